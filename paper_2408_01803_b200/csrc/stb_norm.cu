// Rows between the linears of a decoder block: stb_quantize_i8 (rows in 8 bits, one scale each, the gated activation formed on the way)
// and stb_block_norm (the norms before and after a block with its gate, residual scale and residual sum).
//
// Both are bound by memory: every value is read once and every output written once, whatever happens in between.  A row of up to 1024 values
// belongs to one warp, a longer one to one CTA; row sums and maxima go through shuffles and, per CTA, one barrier each.  With many long rows a
// CTA takes row after row, and the next one's values are on their way into shared memory (cp.async: every thread reads back what it or, fp32,
// its warp has copied, so that the CTA has nothing to wait for) while this one is reduced and written.
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
constexpr int kMaxRowThreads = 1024;
constexpr int kMaxRow = 32768;            // values of a row that fit the registers of a CTA
constexpr int kMaxRowSmem = 224 * 1024;      // dynamic shared memory of a CTA
constexpr float kSmallestMax = 3.0092655e-36f;      // 2^-118: below it 127 / max would overflow; such a row is zeros with scale 0

__host__ __device__ inline int dtype_bytes(int dt) { return dt == STB_F32 ? 4 : 2; }

// ---- two fp32 operations in one instruction ------------------------------------------------------------------------------------------
__device__ __forceinline__ void mul_two(float& d0, float& d1, float a0, float a1, float b0, float b1) {
  asm("{\n\t.reg .b64 a, b;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmul.rn.f32x2 a, a, b;\n\tmov.b64 {%0, %1}, a;\n\t}" : "=f"(d0), "=f"(d1) : "f"(a0), "f"(a1), "f"(b0), "f"(b1));
}
__device__ __forceinline__ void add_two(float& d0, float& d1, float a0, float a1, float b0, float b1) {
  asm("{\n\t.reg .b64 a, b;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tadd.rn.f32x2 a, a, b;\n\tmov.b64 {%0, %1}, a;\n\t}" : "=f"(d0), "=f"(d1) : "f"(a0), "f"(a1), "f"(b0), "f"(b1));
}
__device__ __forceinline__ void fma_two(float& d0, float& d1, float a0, float a1, float b0, float b1, float c0, float c1) {
  asm("{\n\t.reg .b64 a, b, c;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\tfma.rn.f32x2 a, a, b, c;\n\tmov.b64 {%0, %1}, a;\n\t}"
      : "=f"(d0), "=f"(d1) : "f"(a0), "f"(a1), "f"(b0), "f"(b1), "f"(c0), "f"(c1));
}

// ---- a thread's values of a row ------------------------------------------------------------------------------------------------------
// Piece p of thread `lane` of `width` is the eight values at 8 (p width + lane) where rows can be read in 16-byte pieces (their length a multiple
// of 8), else every value is width behind the one before it, so that a warp's loads stay together.
template <bool kVec>
struct RowPlace {
  int lane, width, m;
  __device__ __forceinline__ int at(int p, int k) const { return kVec ? (p * width + lane) * kPiece + k : (p * kPiece + k) * width + lane; }
};
// The element types are arguments of the calls and template arguments of what runs per value: by_type chooses once per row, or, kAll, when the
// kernel is compiled: one 16-bit type for everything is the usual call.
template <int kType> struct TypeOf { static constexpr int value = kType; };
constexpr int kAnyType = -1;
template <int kAll, class F>
__device__ __forceinline__ void by_type(int dt, F f) {
  if constexpr (kAll != kAnyType) f(TypeOf<kAll>{});
  else if (dt == STB_F32) f(TypeOf<STB_F32>{});
  else if (dt == STB_F16) f(TypeOf<STB_F16>{});
  else f(TypeOf<STB_BF16>{});
}
template <int kType>
__device__ __forceinline__ void unpack_two(uint32_t w, float& a, float& b) {
  if (kType == STB_F16) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
    a = f.x; b = f.y;
  } else {
    a = __uint_as_float(w << 16);
    b = __uint_as_float(w & 0xFFFF0000u);
  }
}
template <int kType>
__device__ __forceinline__ uint32_t pack_two(float a, float b) {
  if (kType == STB_F16) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
template <int kType>
__device__ __forceinline__ float load_sixteen(const void* p, size_t i) {
  float a, b;
  unpack_two<kType>(static_cast<const unsigned short*>(p)[i], a, b);
  return a;
}
template <int kType>
__device__ __forceinline__ void unpack_piece(const uint4& a, float (&v)[kPiece]) {
  unpack_two<kType>(a.x, v[0], v[1]); unpack_two<kType>(a.y, v[2], v[3]);
  unpack_two<kType>(a.z, v[4], v[5]); unpack_two<kType>(a.w, v[6], v[7]);
}
// Eight values as they lie in memory: 16 bytes, fp32 twice that, which one instruction moves: two of 16 bytes would each touch half of every 32-byte sector.
template <int kType> struct RawPiece { uint4 w[kType == STB_F32 ? 2 : 1]; };
__device__ __forceinline__ void load_32(const void* p, uint4 (&w)[2]) {
  asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(w[0].x), "=r"(w[0].y), "=r"(w[0].z), "=r"(w[0].w), "=r"(w[1].x), "=r"(w[1].y), "=r"(w[1].z), "=r"(w[1].w) : "l"(p));
}
__device__ __forceinline__ void store_32(void* p, const float (&v)[kPiece]) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               ::"l"(p), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]) : "memory");
}
template <int kType>
__device__ __forceinline__ void values_of(const RawPiece<kType>& r, float (&v)[kPiece]) {
  if constexpr (kType == STB_F32) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      v[4 * h] = __uint_as_float(r.w[h].x); v[4 * h + 1] = __uint_as_float(r.w[h].y); v[4 * h + 2] = __uint_as_float(r.w[h].z); v[4 * h + 3] = __uint_as_float(r.w[h].w);
    }
  } else {
    unpack_piece<kType>(r.w[0], v);
  }
}
// Piece p of the row that starts at `row`: zeros behind its end.  kClamp: values without 16-byte pieces are read at a clamped place, without branches, so that the
// loads of several rows stay together (norms: 1000 x 5111 26 -> 17 us; the quantizer has one row to read and is faster without the clamps, 13 -> 9).
template <int kType, bool kVec, bool kClamp>
__device__ __forceinline__ RawPiece<kType> load_piece(const RowPlace<kVec>& pl, const void* row, int p) {
  RawPiece<kType> r;
  constexpr int kParts = kType == STB_F32 ? 2 : 1;
#pragma unroll
  for (int h = 0; h < kParts; ++h) r.w[h] = make_uint4(0u, 0u, 0u, 0u);
  if constexpr (kVec) {
    const int i = pl.at(p, 0);
    if (i < pl.m) {
      const char* q = static_cast<const char*>(row) + (size_t)i * (2 * kParts);
      if constexpr (kType == STB_F32) load_32(q, r.w);
      else r.w[0] = *reinterpret_cast<const uint4*>(q);
    }
  } else {
    uint32_t u[kPiece];
#pragma unroll
    for (int k = 0; k < kPiece; ++k) {
      const int e = kClamp ? min(pl.at(p, k), pl.m - 1) : pl.at(p, k);
      u[k] = 0u;
      if (kClamp || e < pl.m) u[k] = kType == STB_F32 ? static_cast<const uint32_t*>(row)[e] : (uint32_t)static_cast<const unsigned short*>(row)[e];
    }
    if (kClamp) {
#pragma unroll
      for (int k = 0; k < kPiece; ++k) u[k] = pl.at(p, k) < pl.m ? u[k] : 0u;
    }
    if constexpr (kType == STB_F32) {
      r.w[0] = make_uint4(u[0], u[1], u[2], u[3]);
      r.w[1] = make_uint4(u[4], u[5], u[6], u[7]);
    } else {
      r.w[0] = make_uint4(u[0] | (u[1] << 16), u[2] | (u[3] << 16), u[4] | (u[5] << 16), u[6] | (u[7] << 16));
    }
  }
  return r;
}
// f(p, values) for every piece of the row at `row`, after all of its loads have been asked for.
template <int kAll, int P, bool kVec, class F>
__device__ __forceinline__ void for_row(const RowPlace<kVec>& pl, const void* row, int dt, F f) {
  by_type<kAll>(dt, [&](auto type) {
    constexpr int kType = decltype(type)::value;
    constexpr int kAtOnce = P <= 2 ? P : (!kVec || kType == STB_F32 ? 2 : P);      // (registers)
#pragma unroll
    for (int p0 = 0; p0 < P; p0 += kAtOnce) {
      RawPiece<kType> raw[kAtOnce];
#pragma unroll
      for (int p = 0; p < kAtOnce; ++p) raw[p] = load_piece<kType, kVec, true>(pl, row, p0 + p);
#pragma unroll
      for (int p = 0; p < kAtOnce; ++p) {
        float u[kPiece];
        values_of<kType>(raw[p], u);
        f(p0 + p, u);
      }
    }
  });
}
// A row as it lies in memory, asked for; and, later, f(p, values) for its pieces.
template <int P> struct RawRow { uint4 w[P][2]; };
template <int kAll, int P, bool kVec>
__device__ __forceinline__ void ask_raw(const RowPlace<kVec>& pl, const void* row, int dt, RawRow<P>& raw) {
  by_type<kAll>(dt, [&](auto type) {
    constexpr int kType = decltype(type)::value;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const RawPiece<kType> r = load_piece<kType, kVec, true>(pl, row, p);
      raw.w[p][0] = r.w[0];
      if constexpr (kType == STB_F32) raw.w[p][1] = r.w[1];
    }
  });
}
template <int kAll, int P, class F>
__device__ __forceinline__ void for_raw(const RawRow<P>& raw, int dt, F f) {
  by_type<kAll>(dt, [&](auto type) {
    constexpr int kType = decltype(type)::value;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      RawPiece<kType> r;
      r.w[0] = raw.w[p][0];
      if constexpr (kType == STB_F32) r.w[1] = raw.w[p][1];
      float u[kPiece];
      values_of<kType>(r, u);
      f(p, u);
    }
  });
}
template <int kAll, int P, bool kVec>
__device__ __forceinline__ void store_row(const RowPlace<kVec>& pl, void* row, int dt, const float (&v)[P][kPiece]) {
  by_type<kAll>(dt, [&](auto type) {
    constexpr int kType = decltype(type)::value;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int i = pl.at(p, 0);
      if (kVec && i >= pl.m) break;
      if constexpr (kType == STB_F32) {
        float* q = static_cast<float*>(row);
        if (kVec) {
          store_32(q + i, v[p]);
        } else {
#pragma unroll
          for (int k = 0; k < kPiece; ++k)
            if (pl.at(p, k) < pl.m) q[pl.at(p, k)] = v[p][k];
        }
      } else {
        unsigned short* q = static_cast<unsigned short*>(row);
        uint32_t w[kPiece / 2];
#pragma unroll
        for (int k = 0; k < kPiece / 2; ++k) w[k] = pack_two<kType>(v[p][2 * k], v[p][2 * k + 1]);
        if (kVec) {
          *reinterpret_cast<uint4*>(q + i) = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
#pragma unroll
          for (int k = 0; k < kPiece; ++k)
            if (pl.at(p, k) < pl.m) q[pl.at(p, k)] = (unsigned short)(w[k >> 1] >> (16 * (k & 1)));
        }
      }
    }
  });
}

// ---- pieces on their way -----------------------------------------------------------------------------------------------------------
// A row's pieces in shared memory, in their order: 16-byte part j of piece p of a thread at parts (p width + lane) + j, parts = 1 or, fp32, 2.  Pieces of one
// part a thread copies for itself; those of two the threads of a warp copy for each other, neighbours side by side (each for itself they would take every
// 32-byte sector twice: 4096 x 8192 fp32 in 8 bits 47 us, so 28), and the warp waits for all of its threads' copies.
__device__ __forceinline__ void copy_async16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copy_async_done() {
  asm volatile("cp.async.wait_all;" ::: "memory");
  __syncwarp();
}
template <int kAll, int P>
__device__ __forceinline__ void ask_row(const RowPlace<true>& pl, const void* row, int dt, uint8_t* at) {
  const uint32_t slots = smem_u32(at);
  if ((kAll == kAnyType ? dt : kAll) == STB_F32) {
    __syncwarp();                                   // (the neighbour has read its slots)
    const int lane = pl.lane & 31, first = 2 * (pl.lane - lane) + lane;
#pragma unroll
    for (int p = 0; p < P; ++p) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int part = 2 * p * pl.width + first + 32 * h;
        if (part * 4 < pl.m) copy_async16(slots + (uint32_t)part * 16u, static_cast<const char*>(row) + (size_t)part * 16);
      }
    }
  } else {
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int i = pl.at(p, 0);
      if (i >= pl.m) break;
      copy_async16(slots + (uint32_t)(p * pl.width + pl.lane) * 16u, static_cast<const char*>(row) + (size_t)i * 2);
    }
  }
}
// Zeros in the slots behind the row's end, which nothing is ever copied into (every row ends at the same place).
template <int kAll, int P>
__device__ __forceinline__ void clear_slots(const RowPlace<true>& pl, int dt, uint8_t* slots) {
  const int parts = (kAll == kAnyType ? dt : kAll) == STB_F32 ? 2 : 1;
  for (int p = 0; p < P; ++p)
    for (int h = 0; h < parts; ++h)
      if (pl.at(p, 0) >= pl.m) reinterpret_cast<uint4*>(slots)[parts * (p * pl.width + pl.lane) + h] = make_uint4(0u, 0u, 0u, 0u);
}
template <int kType>
__device__ __forceinline__ RawPiece<kType> slot_raw(const RowPlace<true>& pl, int p, const uint8_t* slots) {
  constexpr int kParts = kType == STB_F32 ? 2 : 1;
  RawPiece<kType> r;
#pragma unroll
  for (int h = 0; h < kParts; ++h) r.w[h] = reinterpret_cast<const uint4*>(slots)[kParts * (p * pl.width + pl.lane) + h];
  return r;
}
// f(p, values) for every piece in the slots
template <int kAll, int P, class F>
__device__ __forceinline__ void for_slots(const RowPlace<true>& pl, int dt, const uint8_t* slots, F f) {
  by_type<kAll>(dt, [&](auto type) {
    constexpr int kType = decltype(type)::value;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      float u[kPiece];
      values_of<kType>(slot_raw<kType>(pl, p, slots), u);
      f(p, u);
    }
  });
}

// ---- sums and maxima over the threads of a row ----------------------------------------------------------------------------------------
// kWarp: the row belongs to this warp.  Else to the CTA: every reduction of a kernel has a `slot` of its own in shared memory, so that one
// barrier does for each.  All orders are fixed.
template <bool kWarp>
__device__ __forceinline__ float row_sum(float v, float (*part)[32], int slot) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
  if (kWarp) return v;
  const int lane = threadIdx.x & 31;
  if (lane == 0) part[slot][threadIdx.x >> 5] = v;
  __syncthreads();
  v = lane < (int)(blockDim.x >> 5) ? part[slot][lane] : 0.0f;
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
  return v;
}
// of the magnitudes' bit patterns: an infinity is above every number and a NaN above that
template <bool kWarp>
__device__ __forceinline__ uint32_t row_max(uint32_t v, float (*part)[32], int slot) {
  v = __reduce_max_sync(0xFFFFFFFFu, v);
  if (kWarp) return v;
  const int lane = threadIdx.x & 31;
  if (lane == 0) part[slot][threadIdx.x >> 5] = __uint_as_float(v);
  __syncthreads();
  v = lane < (int)(blockDim.x >> 5) ? __float_as_uint(part[slot][lane]) : 0u;
  return __reduce_max_sync(0xFFFFFFFFu, v);
}
// the largest of three, and of three a NaN if one is; the smallest of three
__device__ __forceinline__ float max3(float a, float b, float c) {
  asm("max.f32 %0, %0, %1, %2;" : "+f"(a) : "f"(b), "f"(c));
  return a;
}
__device__ __forceinline__ float max3_nan(float a, float b, float c) {
  asm("max.NaN.f32 %0, %0, %1, %2;" : "+f"(a) : "f"(b), "f"(c));
  return a;
}
__device__ __forceinline__ float min3(float a, float b, float c) {
  asm("min.f32 %0, %0, %1, %2;" : "+f"(a) : "f"(b), "f"(c));
  return a;
}
template <int P>
__device__ __forceinline__ uint32_t max_bits(const float (&v)[P][kPiece]) {
  float b = 0.0f;
#pragma unroll
  for (int p = 0; p < P; ++p)
#pragma unroll
    for (int k = 0; k < kPiece; k += 2) b = max3_nan(b, fabsf(v[p][k]), fabsf(v[p][k + 1]));
  return __float_as_uint(b);
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
// The whole number nearest to 127 v / largest, decided between two neighbours by exact products where v inverse lies next to the border between them.
__device__ __forceinline__ uint32_t value_i8_exact(float v, float inverse, float largest) {
  const float t = v * inverse;
  float r = rintf(t);
  if (fabsf(t - r) > 0.4999f) {
    const float k = floorf(fabsf(t));
    const double a = 254.0 * (double)fabsf(v), c = (2.0 * (double)k + 1.0) * (double)largest;      // both exact
    r = copysignf(a > c ? k + 1.0f : (a < c ? k : 2.0f * rintf(0.5f * (k + 0.25f))), v);           // the even one of k, k + 1 on the border itself
  }
  return (uint32_t)(int)r & 0xFFu;
}
__device__ __noinline__ uint2 piece_i8_exact(float4 a, float4 b, float inverse, float largest) {
  const float v[kPiece] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
  uint2 q = make_uint2(0u, 0u);
#pragma unroll
  for (int k = 0; k < kPiece; ++k) (k < 4 ? q.x : q.y) |= value_i8_exact(v[k], inverse, largest) << (8 * (k & 3));
  return q;
}
constexpr float kRoundBias = 12582912.0f;           // 1.5 * 2^23: adding it rounds to the nearest whole number, whose low byte is the sum's
template <bool kVec>
__device__ __forceinline__ void store_piece_i8(const RowPlace<kVec>& pl, int8_t* row, int p, const float (&v)[kPiece], const RowScale& s) {
  uint32_t q[kPiece];
  float off = 0.0f;                                 // the farthest from a whole number: 0.5 is a border
#pragma unroll
  for (int k = 0; k < kPiece; k += 2) {
    float u0, u1, r0, r1, d0, d1;
    fma_two(u0, u1, v[k], v[k + 1], s.inverse, s.inverse, kRoundBias, kRoundBias);
    add_two(r0, r1, u0, u1, -kRoundBias, -kRoundBias);
    fma_two(d0, d1, v[k], v[k + 1], -s.inverse, -s.inverse, r0, r1);
    off = max3(off, fabsf(d0), fabsf(d1));
    q[k] = __float_as_uint(u0);
    q[k + 1] = __float_as_uint(u1);
  }
  uint2 two = make_uint2(__byte_perm(__byte_perm(q[0], q[1], 0x0040), __byte_perm(q[2], q[3], 0x0040), 0x5410),
                         __byte_perm(__byte_perm(q[4], q[5], 0x0040), __byte_perm(q[6], q[7], 0x0040), 0x5410));
  if (off > 0.4999f) two = piece_i8_exact(make_float4(v[0], v[1], v[2], v[3]), make_float4(v[4], v[5], v[6], v[7]), s.inverse, s.largest);
  if (s.inverse == 0.0f) two = make_uint2(0u, 0u);  // (infinities and NaN among the values)
  if (kVec) {
    *reinterpret_cast<uint2*>(row + pl.at(p, 0)) = two;
  } else {
#pragma unroll
    for (int k = 0; k < kPiece; ++k)
      if (pl.at(p, k) < pl.m) row[pl.at(p, k)] = (int8_t)(((k < 4 ? two.x : two.y) >> (8 * (k & 3))) & 0xFFu);
  }
}
template <int P, bool kVec>
__device__ __forceinline__ void store_row_i8(const RowPlace<kVec>& pl, int8_t* row, const float (&v)[P][kPiece], const RowScale& s) {
#pragma unroll
  for (int p = 0; p < P; ++p) {
    if (pl.at(p, 0) >= pl.m) break;
    store_piece_i8<kVec>(pl, row, p, v[p], s);
  }
}

// the larger magnitude of each half (a holds magnitudes; a NaN stays one)
template <int kType>
__device__ __forceinline__ uint32_t max_magnitudes(uint32_t a, uint32_t b) {
  if (kType == STB_F16) {
    const __half2 r = __hmax2_nan(*reinterpret_cast<const __half2*>(&a), __habs2(*reinterpret_cast<const __half2*>(&b)));
    return *reinterpret_cast<const uint32_t*>(&r);
  }
  const __nv_bfloat162 r = __hmax2_nan(*reinterpret_cast<const __nv_bfloat162*>(&a), __habs2(*reinterpret_cast<const __nv_bfloat162*>(&b)));
  return *reinterpret_cast<const uint32_t*>(&r);
}

// ---- the gated activation ---------------------------------------------------------------------------------------------------------
// silu(a) b rounded to fp32 and then to the 16-bit type, as exact arithmetic would.  In fp32 it is known within (5 + 0.75 |min(a, 0)|) 2^-23 (in units of
// 2^-23: the power of two 2 by its specification and 0.75 |a| from its rounded argument, of which e / (1 + e) reaches the result, the reciprocal 1,
// the sum, the two products and the fp32 rounding half a one each; a >= -80, where nothing leaves fp32's range): both ends of a band somewhat wider, of
// one width for the eight values of a piece, are rounded, and nearly always give the same 16-bit value.  Where they do not, that of the smaller magnitude is
// kept, the other is the next one up, and the value is marked: it is evaluated in float64 only where the choice would show, in the row's largest magnitude
// or in the value's 8 bits.  (Everything in float64 would be 150 instructions a value.)
template <int kType>
__device__ __noinline__ uint32_t gated_exact(float a0, float a1, float b0, float b1) {
  const double d0 = (double)a0, d1 = (double)a1;
  return pack_two<kType>((float)(d0 / (1.0 + exp(-d0)) * (double)b0), (float)(d1 / (1.0 + exp(-d1)) * (double)b1));
}
constexpr float kUlp = 1.1920929e-7f;               // 2^-23
__device__ __forceinline__ float gated_band(float least) { return fmaf(fminf(least, 0.0f), -kUlp, 6.0f * kUlp); }
template <int kType>
__device__ __forceinline__ void gated_two(float a0, float a1, float b0, float b1, float band, uint32_t& lo, uint32_t& hi) {
  float t0, t1, h0, h1, l0, l1, m0, m1;
  mul_two(t0, t1, a0, a1, -1.4426950408889634f, -1.4426950408889634f);
  asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(t0));
  asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(t1));
  add_two(t0, t1, t0, t1, 1.0f, 1.0f);
  asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(t0));
  asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(t1));
  mul_two(h0, h1, a0, a1, t0, t1);
  mul_two(h0, h1, h0, h1, b0, b1);
  fma_two(m0, m1, h0, h1, band, band, h0, h1);
  fma_two(l0, l1, h0, h1, -band, -band, h0, h1);
  lo = pack_two<kType>(l0, l1);
  hi = pack_two<kType>(m0, m1);
}

// ---- stb_quantize_i8 ----------------------------------------------------------------------------------------------------------------
struct QuantI8Args {
  const void *x, *x2;
  int rows, m;
  size_t ldx, ldx2, ldq;
  int8_t* q;
  float* scale;
};
// The values: of kType as they are, or (16-bit types) gated.  What a thread holds of a row between its largest magnitude and its 8 bits.  Gated values: h is
// the candidate of smaller magnitude, marks says which have two: bits 4 (p % 4) + k and 16 beyond it of word p / 4 the two values of pair k of piece p.
template <int P, int kType> struct QuantRow {
  uint32_t h[P][kPiece / 2], marks[(P + 3) / 4];
  __device__ __forceinline__ uint32_t marks_of(int p) const { return (marks[p / 4] >> (4 * (p & 3))) & 0x000F000Fu; }
};
template <int P> struct QuantRow<P, STB_F32> { float v[P][kPiece]; };

// Settles the marked values of a piece: in float64, from the inputs again, where the 8 bits depend on which of the two candidates it is (a magnitude's next
// one up: its bits plus one), or, inverse < 0, all of them.  The values lie at `at`, each `step` behind the one before it.
template <int kType>
__device__ __noinline__ uint4 settle_piece(uint4 h, uint32_t marks, const void* xr, const void* xr2, int at, int step, int m, float inverse, float largest) {
#pragma unroll
  for (int k = 0; k < kPiece / 2; ++k) {
    uint32_t& two = k == 0 ? h.x : (k == 1 ? h.y : (k == 2 ? h.z : h.w));
    const uint32_t here = (marks >> k) & 0x00010001u;
    if (here == 0u) continue;
    bool shows = inverse < 0.0f;
    if (!shows) {
      float a, b, c, d;
      unpack_two<kType>(two, a, b);
      unpack_two<kType>(two + here, c, d);
      shows = value_i8_exact(a, inverse, largest) != value_i8_exact(c, inverse, largest) || value_i8_exact(b, inverse, largest) != value_i8_exact(d, inverse, largest);
    }
    const int i = at + 2 * k * step, j = i + step;
    if (shows) {
      const float a0 = i < m ? load_sixteen<kType>(xr, (size_t)i) : 0.0f, b0 = i < m ? load_sixteen<kType>(xr2, (size_t)i) : 0.0f;
      const float a1 = j < m ? load_sixteen<kType>(xr, (size_t)j) : 0.0f, b1 = j < m ? load_sixteen<kType>(xr2, (size_t)j) : 0.0f;
      two = gated_exact<kType>(a0, a1, b0, b1);
    }
  }
  return h;
}
template <int kType>
__device__ __noinline__ uint4 gated_exact_piece(uint4 ra, uint4 rb) {
  float a[kPiece], b[kPiece];
  unpack_piece<kType>(ra, a);
  unpack_piece<kType>(rb, b);
  return make_uint4(gated_exact<kType>(a[0], a[1], b[0], b[1]), gated_exact<kType>(a[2], a[3], b[2], b[3]), gated_exact<kType>(a[4], a[5], b[4], b[5]), gated_exact<kType>(a[6], a[7], b[6], b[7]));
}
__device__ __forceinline__ uint32_t one_where_any(uint32_t halves) {      // 1 in every half that is not zero
  uint32_t r;
  asm("min.u16x2 %0, %1, %2;" : "=r"(r) : "r"(halves), "r"(0x00010001u));
  return r;
}
// The gated values of a piece.  low, top: per half the largest magnitude of the smaller candidates and of the larger ones.
template <int P, int kType>
__device__ __forceinline__ void gate_piece(QuantRow<P, kType>& r, int p, const uint4& ra, const uint4& rb, uint32_t& low, uint32_t& top) {
  float a[kPiece], b[kPiece];
  unpack_piece<kType>(ra, a);
  unpack_piece<kType>(rb, b);
  uint32_t lo[kPiece / 2], hi[kPiece / 2];
  float least = a[0];
#pragma unroll
  for (int k = 1; k + 1 < kPiece; k += 2) least = min3(least, a[k], a[k + 1]);
  least = fminf(least, a[kPiece - 1]);
  const float band = gated_band(least);
#pragma unroll
  for (int k = 0; k < kPiece / 2; ++k) gated_two<kType>(a[2 * k], a[2 * k + 1], b[2 * k], b[2 * k + 1], band, lo[k], hi[k]);
  if (least < -80.0f) {
    const uint4 e = gated_exact_piece<kType>(ra, rb);
    lo[0] = hi[0] = e.x; lo[1] = hi[1] = e.y; lo[2] = hi[2] = e.z; lo[3] = hi[3] = e.w;
  }
#pragma unroll
  for (int k = 0; k < kPiece / 2; ++k) {
    r.h[p][k] = lo[k];
    r.marks[p / 4] += one_where_any((lo[k] ^ hi[k]) & 0x7FFF7FFFu) * (1u << (4 * (p & 3) + k));      // (a zero's sign says nothing)
    low = max_magnitudes<kType>(low, lo[k]);
    top = max_magnitudes<kType>(top, hi[k]);
  }
}
// fp32 bits of a 16-bit magnitude
template <int kType>
__device__ __forceinline__ uint32_t magnitude_bits(uint32_t m) {
  float a, b;
  unpack_two<kType>(m, a, b);
  return __float_as_uint(a);
}
// kWarp: a row belongs to a warp, else to the CTA, which takes every gridDim-th one.  kAsync: the pieces of the next row are on their way.
// Measured: 11008 x 4096 fp16 22.8 us (5.9 TB/s), 4096 x 28672 fp32 91 us (6.5 TB/s), bound by HBM; gated 2048 x 28672 bf16 72.5 us (4.1 TB/s), bound by the way through a row:
// one CTA of 896 threads an SM has nothing to issue around its barrier (issue active 63 %, no pipe above 50 %; 28 instructions a value); 1 x 4096 1.6 us, the launch.
template <int P, int kType, bool kGated, bool kVec, bool kWarp, bool kAsync>
__global__ void __launch_bounds__(kWarp ? 256 : (kAsync ? (kGated ? kMaxRowThreads : 512) : (!kVec && P > 2 ? 512 : kMaxRowThreads)),
                                  kWarp || (kAsync && !kGated && (P <= 4 || kType != STB_F32)) || (!kVec && P == 4) ? 2 : 1)
quantize_i8_kernel(const QuantI8Args args) {
  extern __shared__ __align__(16) uint8_t slots[];
  __shared__ float sh[4][32];                       // the parts of a row's two reductions, and of the next one's
  const void *x = args.x, *x2 = args.x2;
  begin_after(x, x2);
  constexpr int kBytes = kType == STB_F32 ? 4 : 2;
  // (unsigned: a row behind the last one is below 2^32, whatever their number)
  const uint32_t rows = (uint32_t)args.rows, stride = kWarp ? gridDim.x * (blockDim.x >> 5) : gridDim.x;
  uint32_t row = kWarp ? blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5) : blockIdx.x;
  int slot = 0;
  const RowPlace<kVec> pl{kWarp ? (int)(threadIdx.x & 31) : (int)threadIdx.x, kWarp ? 32 : (int)blockDim.x, args.m};
  uint8_t *slot_x = slots, *slot_x2 = slots + (size_t)(P * pl.width) * 16u;
  auto row_x = [&](uint32_t r) { return static_cast<const char*>(x) + (size_t)r * args.ldx * kBytes; };
  auto row_x2 = [&](uint32_t r) { return static_cast<const char*>(x2) + (size_t)r * args.ldx2 * kBytes; };
  auto ask = [&](uint32_t r) {
    if constexpr (kAsync) {
      ask_row<kType, P>(pl, row_x(r), kType, slot_x);
      if (kGated) ask_row<kType, P>(pl, row_x2(r), kType, slot_x2);
    }
  };
  auto settle = [&](QuantRow<P, kType>& r, int p, float inverse, float largest) {
    if constexpr (kGated) {
      const uint4 h = settle_piece<kType>(make_uint4(r.h[p][0], r.h[p][1], r.h[p][2], r.h[p][3]), r.marks_of(p), row_x(row), row_x2(row), pl.at(p, 0), pl.at(0, 1) - pl.at(0, 0), args.m,
                                          inverse, largest);
      r.h[p][0] = h.x; r.h[p][1] = h.y; r.h[p][2] = h.z; r.h[p][3] = h.w;
    }
  };
  if constexpr (kAsync) {
    clear_slots<kType, P>(pl, kType, slot_x);
    if (kGated) clear_slots<kType, P>(pl, kType, slot_x2);
    if (row < rows) ask(row);
  }
  for (; row < rows; row += stride, slot ^= 2) {
    QuantRow<P, kType> r;
    if constexpr (kGated) {
#pragma unroll
      for (int i = 0; i < (P + 3) / 4; ++i) r.marks[i] = 0;
    }
    uint32_t bits;
    if constexpr (kAsync) copy_async_done();
    RawPiece<kType> raw[P], raw2[kGated && !kAsync ? P : 1];
    if constexpr (!kAsync) {
#pragma unroll
      for (int p = 0; p < P; ++p) {
        raw[p] = load_piece<kType, kVec, false>(pl, row_x(row), p);
        if constexpr (kGated) raw2[p] = load_piece<kType, kVec, false>(pl, row_x2(row), p);
      }
    }
    if constexpr (kType == STB_F32) {
#pragma unroll
      for (int p = 0; p < P; ++p) {
        if constexpr (kAsync) raw[p] = slot_raw<kType>(pl, p, slot_x);
        values_of<kType>(raw[p], r.v[p]);
      }
      bits = row_max<kWarp>(max_bits<P>(r.v), sh, slot);
    } else {
      uint32_t top = 0, low = 0;
#pragma unroll
      for (int p = 0; p < P; ++p) {
        if constexpr (kAsync) raw[p] = slot_raw<kType>(pl, p, slot_x);
        if constexpr (kGated) {
          if constexpr (kAsync) raw2[0] = slot_raw<kType>(pl, p, slot_x2);
          gate_piece<P, kType>(r, p, raw[p].w[0], raw2[kAsync ? 0 : p].w[0], low, top);
        } else {
          r.h[p][0] = raw[p].w[0].x; r.h[p][1] = raw[p].w[0].y; r.h[p][2] = raw[p].w[0].z; r.h[p][3] = raw[p].w[0].w;
#pragma unroll
          for (int k = 0; k < kPiece / 2; ++k) top = max_magnitudes<kType>(top, r.h[p][k]);
        }
      }
      uint32_t largest = max(top >> 16, top & 0xFFFFu);
      if constexpr (kGated) {
        // The largest of the larger candidates and, behind it, that of the smaller ones (of the threads that have the former): the same, or else the
        // largest magnitude itself has two candidates.
        largest = row_max<kWarp>((largest << 16) | max(low >> 16, low & 0xFFFFu), sh, slot);
        const bool unsettled = (largest >> 16) != (largest & 0xFFFFu);      // (for every thread of the row alike)
        largest >>= 16;
        if (unsettled) {
          top = 0;
#pragma unroll
          for (int p = 0; p < P; ++p) {
            if (r.marks_of(p)) settle(r, p, -1.0f, 0.0f);
#pragma unroll
            for (int k = 0; k < kPiece / 2; ++k) top = max_magnitudes<kType>(top, r.h[p][k]);
          }
#pragma unroll
          for (int i = 0; i < (P + 3) / 4; ++i) r.marks[i] = 0;
          largest = row_max<kWarp>(max(top >> 16, top & 0xFFFFu), sh, slot + 1);
        }
      } else {
        largest = row_max<kWarp>(largest, sh, slot);
      }
      bits = magnitude_bits<kType>(largest);
    }
    if (kAsync && row + stride < rows) ask(row + stride);        // (this row's pieces have been read: its largest magnitude is known)
    const RowScale s = row_scale(bits);
    int8_t* qr = args.q + (size_t)row * args.ldq;
    if (pl.lane == 0) args.scale[row] = s.scale;
    if constexpr (kType == STB_F32) {
      store_row_i8<P, kVec>(pl, qr, r.v, s);
    } else {
#pragma unroll
      for (int p = 0; p < P; ++p) {
        if (pl.at(p, 0) >= pl.m) break;
        float v[kPiece];
        unpack_piece<kType>(make_uint4(r.h[p][0], r.h[p][1], r.h[p][2], r.h[p][3]), v);
        if (kGated && r.marks_of(p)) {
          // only a value that lies within a step of the 16-bit type of a border needs to be settled: 2^-10 (fp16) or 2^-7 of it, and 2^-24 (fp16) where that is less
          constexpr float kStep = kType == STB_F16 ? 9.765625e-4f : 7.8125e-3f;
          float near = 0.0f;
#pragma unroll
          for (int k = 0; k < kPiece; ++k) {
            const float t = v[k] * s.inverse;
            near = fmaxf(near, fmaf(fabsf(t), kStep, fabsf(t - rintf(t))));
          }
          if (near > 0.4998f - 6.0e-8f * s.inverse) {
            settle(r, p, s.inverse, s.largest);
            unpack_piece<kType>(make_uint4(r.h[p][0], r.h[p][1], r.h[p][2], r.h[p][3]), v);
          }
        }
        store_piece_i8<kVec>(pl, qr, p, v, s);
      }
    }
  }
}
// A row that does not fit the registers of a CTA is read twice.
template <int kType, bool kGated, bool kVec>
__global__ void __launch_bounds__(kMaxRowThreads)
quantize_i8_long_kernel(const QuantI8Args args) {
  __shared__ float sh[1][32];
  const void *x = args.x, *x2 = args.x2;
  begin_after(x, x2);
  constexpr int kBytes = kType == STB_F32 ? 4 : 2, kSpan = kMaxRowThreads * kPiece;
  const int row = (int)blockIdx.x;
  const char *xr = static_cast<const char*>(x) + (size_t)row * args.ldx * kBytes, *xr2 = static_cast<const char*>(x2) + (size_t)row * args.ldx2 * kBytes;
  RowPlace<kVec> pl{(int)threadIdx.x, kMaxRowThreads, args.m};
  float v[1][kPiece];
  auto read = [&](int base) {
    pl.m = args.m - base;
    values_of<kType>(load_piece<kType, kVec, false>(pl, xr + (size_t)base * kBytes, 0), v[0]);
    if constexpr (kGated) {
      float b[kPiece];
      values_of<kType>(load_piece<kType, kVec, false>(pl, xr2 + (size_t)base * kBytes, 0), b);
#pragma unroll
      for (int k = 0; k < kPiece; k += 2) {
        uint32_t lo, hi;
        const float least = fminf(v[0][k], v[0][k + 1]);
        gated_two<kType>(v[0][k], v[0][k + 1], b[k], b[k + 1], gated_band(least), lo, hi);
        if (lo != hi || least < -80.0f) lo = gated_exact<kType>(v[0][k], v[0][k + 1], b[k], b[k + 1]);
        unpack_two<kType>(lo, v[0][k], v[0][k + 1]);
      }
    }
  };
  uint32_t bits = 0;
  for (int base = 0;; base += kSpan) { read(base); bits = max(bits, max_bits<1>(v)); if (args.m - base <= kSpan) break; }
  const RowScale s = row_scale(row_max<false>(bits, sh, 0));
  if (threadIdx.x == 0) args.scale[row] = s.scale;
  for (int base = 0;; base += kSpan) {
    read(base);
    store_row_i8<1, kVec>(pl, args.q + (size_t)row * args.ldq + base, v, s);
    if (args.m - base <= kSpan) break;
  }
}

// ---- stb_block_norm -----------------------------------------------------------------------------------------------------------------
template <int P, bool kVec, bool kWarp>
__device__ __forceinline__ void norm_row(const RowPlace<kVec>& pl, float (&v)[P][kPiece], int kind, float eps, float (*sh)[32], int slot) {
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
  float even = 0.0f, odd = 0.0f;
#pragma unroll
  for (int p = 0; p < P; ++p)
#pragma unroll
    for (int k = 0; k < kPiece; k += 2) fma_two(even, odd, v[p][k], v[p][k + 1], v[p][k], v[p][k + 1], even, odd);
  const float inv = rsqrtf(fmaf(row_sum<kWarp>(even + odd, sh, slot + 1), per, eps));
#pragma unroll
  for (int p = 0; p < P; ++p)
#pragma unroll
    for (int k = 0; k < kPiece; k += 2) mul_two(v[p][k], v[p][k + 1], v[p][k], v[p][k + 1], inv, inv);
}
// What bounds it: HBM with one norm and 16 bits out (4096 x 4096 fp16 20.5 us, 6.5 TB/s); issue and the reductions of a row with more (to 8 bits 22.4 us, 5.3 TB/s; the
// norms before and after the sum, 2048 x 8192 bf16, 27.9 us, 4.8 TB/s); the launch and one trip to HBM for a token (4096 values 2.1 us).
// kAll: the type of x, the residual and the weights, where it is the same 16-bit type.  kRoomy (kAsync, four pieces): 80 registers a thread, of which 768 fit an
// SM, instead of 64 and 1024.
template <int kAll, int P, bool kVec, bool kWarp, bool kAsync, bool kRoomy = false>
__global__ void __launch_bounds__(kWarp ? 256 : (kRoomy ? 768 : (kAsync || (!kVec && P > 2) ? 512 : kMaxRowThreads)), kWarp || (kAsync && P <= 4 && !kRoomy) ? 2 : 1)
block_norm_kernel(const __grid_constant__ stb_norm a) {
  extern __shared__ __align__(16) uint8_t slots[];
  __shared__ float sh[10][32];                      // the parts of a row's five reductions, and of the next one's
  const void *x = a.x, *resid = a.resid, *pw = a.post_weight, *pb = a.post_bias, *gate = a.gate, *w = a.weight, *b = a.bias;
  begin_after(x, resid, pw, pb, gate, w, b);
  // (unsigned: a row behind the last one is below 2^32, whatever their number)
  const uint32_t rows = (uint32_t)a.tokens, stride = kWarp ? gridDim.x * (blockDim.x >> 5) : gridDim.x;
  uint32_t row = kWarp ? blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5) : blockIdx.x;
  int slot = 0;
  const RowPlace<kVec> pl{kWarp ? (int)(threadIdx.x & 31) : (int)threadIdx.x, kWarp ? 32 : (int)blockDim.x, a.h};
  auto row_of = [&](const void* base, size_t r, size_t ld, int dt) { return static_cast<const char*>(base) + r * ld * (size_t)dtype_bytes(dt); };
  uint8_t *slot_x = slots, *slot_r = slots + (size_t)(P * pl.width) * ((kAll == kAnyType ? a.xdt : kAll) == STB_F32 ? 32u : 16u);
  auto ask = [&](uint32_t r) {
    if constexpr (kAsync) {
      ask_row<kAll, P>(pl, row_of(x, r, a.ldx, a.xdt), a.xdt, slot_x);
      if (resid) ask_row<kAll, P>(pl, row_of(resid, r, a.ldr, a.rdt), a.rdt, slot_r);
    }
  };
  if constexpr (kAsync) {
    clear_slots<kAll, P>(pl, a.xdt, slot_x);
    if (resid) clear_slots<kAll, P>(pl, a.rdt, slot_r);
    if (row < rows) ask(row);
  }
  for (; row < rows; row += stride, slot ^= 5) {
    // What is asked for before the first sum: the residual beside x, and the vectors, as far as registers hold them.
    constexpr bool kEarly = !kAsync && (kWarp || P <= 2), kAhead = kVec && !kAsync && (P == 1 || (P == 2 && kAll != kAnyType));
    float v[P][kPiece];
    RawRow<kEarly ? P : 1> raw_r;
    RawRow<kAhead ? P : 1> raw_pw, raw_gate, raw_w;
    const char* gate_row = row_of(gate, gate ? row / (uint32_t)a.tokens_per_gate : 0u, a.ldgate, a.wdt);
    auto take = [&](int p, const float (&u)[kPiece]) {
#pragma unroll
      for (int k = 0; k < kPiece; ++k) v[p][k] = u[k];
    };
    auto times = [&](int p, const float (&u)[kPiece]) {
#pragma unroll
      for (int k = 0; k < kPiece; k += 2) mul_two(v[p][k], v[p][k + 1], v[p][k], v[p][k + 1], u[k], u[k + 1]);
    };
    auto plus = [&](int p, const float (&u)[kPiece]) {
#pragma unroll
      for (int k = 0; k < kPiece; k += 2) add_two(v[p][k], v[p][k + 1], v[p][k], v[p][k + 1], u[k], u[k + 1]);
    };
    auto onto = [&](int p, const float (&u)[kPiece]) {
#pragma unroll
      for (int k = 0; k < kPiece; k += 2) fma_two(v[p][k], v[p][k + 1], v[p][k], v[p][k + 1], a.alpha, a.alpha, u[k], u[k + 1]);
    };
    if constexpr (kAsync) {
      copy_async_done();
      for_slots<kAll, P>(pl, a.xdt, slot_x, take);
    } else if constexpr (kEarly) {
      RawRow<P> raw_x;
      ask_raw<kAll, P, kVec>(pl, row_of(x, row, a.ldx, a.xdt), a.xdt, raw_x);
      if (resid) ask_raw<kAll, P, kVec>(pl, row_of(resid, row, a.ldr, a.rdt), a.rdt, raw_r);
      if constexpr (kAhead) {
        if (pw) ask_raw<kAll, P, kVec>(pl, pw, a.wdt, raw_pw);
        if (gate) ask_raw<kAll, P, kVec>(pl, gate_row, a.wdt, raw_gate);
        if (w) ask_raw<kAll, P, kVec>(pl, w, a.wdt, raw_w);
      }
      for_raw<kAll, P>(raw_x, a.xdt, take);
    } else {
      for_row<kAll, P, kVec>(pl, row_of(x, row, a.ldx, a.xdt), a.xdt, take);
    }
    if (a.post) {
      norm_row<P, kVec, kWarp>(pl, v, a.kind, a.eps, sh, slot);
      if constexpr (kAhead) {
        if (pw) for_raw<kAll, P>(raw_pw, a.wdt, times);
      } else {
        if (pw) for_row<kAll, P, kVec>(pl, pw, a.wdt, times);
      }
      if (pb) for_row<kAll, P, kVec>(pl, pb, a.wdt, plus);
    }
    if constexpr (kAhead) {
      if (gate) for_raw<kAll, P>(raw_gate, a.wdt, times);
    } else {
      if (gate) for_row<kAll, P, kVec>(pl, gate_row, a.wdt, times);
    }
    if (!resid) {
#pragma unroll
      for (int p = 0; p < P; ++p)
#pragma unroll
        for (int k = 0; k < kPiece; ++k) v[p][k] *= a.alpha;
    } else if constexpr (kEarly) {
      for_raw<kAll, P>(raw_r, a.rdt, onto);
    } else if constexpr (kAsync) {
      for_slots<kAll, P>(pl, a.rdt, slot_r, onto);
    } else {
      for_row<kAll, P, kVec>(pl, row_of(resid, row, a.ldr, a.rdt), a.rdt, onto);
    }
    if (a.resid_out) store_row<kAll, P, kVec>(pl, const_cast<char*>(row_of(a.resid_out, row, a.ldro, a.rdt)), a.rdt, v);
    const bool more = kAsync && row + stride < rows;
    if (!a.y && !a.q) {
      if (more) ask(row + stride);
      continue;
    }
    norm_row<P, kVec, kWarp>(pl, v, a.kind, a.eps, sh, slot + 2);
    if (more) ask(row + stride);                   // (this row's pieces have been read: its sum is known)
    if constexpr (kAhead) {
      if (w) for_raw<kAll, P>(raw_w, a.wdt, times);
    } else {
      if (w) for_row<kAll, P, kVec>(pl, w, a.wdt, times);
    }
    if (b) for_row<kAll, P, kVec>(pl, b, a.wdt, plus);
    if (a.y) store_row<kAnyType, P, kVec>(pl, const_cast<char*>(row_of(a.y, row, a.ldy, a.ydt)), a.ydt, v);
    if (a.q) {
      const RowScale s = row_scale(row_max<kWarp>(max_bits<P>(v), sh, slot + 4));
      if (pl.lane == 0) a.q_scale[row] = s.scale;
      store_row_i8<P, kVec>(pl, a.q + (size_t)row * a.ldq, v, s);
    }
  }
}

// ---- launches -----------------------------------------------------------------------------------------------------------------------
// How rows of m values are dealt out.
//   warp:    rows of up to 256 values, or of up to 1024 where there are more than SMs; 1, 2 or 4 pieces per lane
//   slots:   the next row on its way into shared memory: more than 296 rows that can be read in 16-byte pieces, 4 or 8 pieces per thread, whichever fills
//            an SM better (resident4, resident8: the threads that its registers take; most4: a CTA's with 4), as many CTAs as stay on the GPU
//   else:    one CTA per row, with one piece per thread as long as 1024 threads reach, for the shortest way through a row; `any_pieces` of them where there are
//            many rows and no 16-byte pieces, for more rows at a time
struct RowShape { bool warp, slots, longer; int pieces, threads, grid; uint32_t smem; };
struct RowNeeds { uint32_t piece_bytes, static_smem; int resident4, resident8, most4, any_pieces; };
static RowShape row_shape(int m, int rows, bool vec, const RowNeeds& need) {
  RowShape s = {};
  const int pieces = (m + kPiece - 1) / kPiece;
  if (m > kMaxRow) { s.longer = true; s.pieces = 1; s.threads = kMaxRowThreads; s.grid = rows; return s; }
  if (m <= 256 || (m <= 1024 && rows > 148)) {
    const int per_cta = rows >= 148 * 8 ? 8 : (rows >= 148 * 2 ? 2 : 1);
    s.warp = true;
    s.pieces = pieces <= 32 ? 1 : (pieces <= 64 ? 2 : 4);
    s.threads = 32 * per_cta;
    s.grid = (int)(((long long)rows + per_cta - 1) / per_cta);
    return s;
  }
  if (vec && rows > 296) {
    const int threads4 = ((pieces + 3) / 4 + 31) / 32 * 32, threads8 = ((pieces + 7) / 8 + 31) / 32 * 32;
    const bool four = threads4 <= need.most4 && need.resident4 / threads4 * threads4 >= need.resident8 / threads8 * threads8;      // threads that an SM holds
    s.pieces = four ? 4 : 8;
    s.threads = four ? threads4 : threads8;
    s.smem = (uint32_t)(s.pieces * s.threads) * need.piece_bytes;
    if (s.smem <= (uint32_t)kMaxRowSmem) {          // (not two inputs of fp32 beyond 28672 values)
      int resident = (four ? need.resident4 : need.resident8) / s.threads, by_smem = (int)(228u * 1024u / (s.smem + 1024u + need.static_smem));
      if (resident > by_smem) resident = by_smem;
      if (resident < 1) resident = 1;
      s.slots = true;
      s.grid = rows < 148 * resident ? rows : 148 * resident;
      return s;
    }
    s.smem = 0;
  }
  s.pieces = pieces <= kMaxRowThreads ? 1 : (pieces <= 2 * kMaxRowThreads ? 2 : (vec ? 4 : 8));
  if (!vec && rows > 148 && s.pieces < need.any_pieces) s.pieces = need.any_pieces;
  s.threads = ((pieces + s.pieces - 1) / s.pieces + 31) / 32 * 32;
  s.grid = rows;
  return s;
}

// a piece's bytes: 8 bits 8, 16 bits 16, fp32 32
static bool rows_aligned(const void* p, size_t ld, int bytes, size_t to) { return !p || ((reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0 && (ld * (size_t)bytes) % to == 0); }
static bool element_aligned(const void* p, int dt) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(dtype_bytes(dt) - 1)) == 0; }
static bool known_dtype(int dt) { return dt == STB_F16 || dt == STB_BF16 || dt == STB_F32; }

// A kernel with more than 48 KB of shared memory (what it declares included) has to be allowed it, on every device.
template <auto kKernel, typename A>
static cudaError_t launch_rows(const RowShape& s, cudaStream_t st, const A& args) {
  if (s.smem > 46 * 1024) {
    static bool done[64] = {};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64 || !done[dev]) {
      e = cudaFuncSetAttribute(kKernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxRowSmem);
      if (e != cudaSuccess) return e;
      if (dev >= 0 && dev < 64) done[dev] = true;
    }
  }
  return launch_after(kKernel, dim3((unsigned)s.grid), dim3((unsigned)s.threads), s.smem, st, args);
}

template <int kType, bool kGated, bool kVec>
static cudaError_t launch_quantize_as(const QuantI8Args& a, const RowShape& s, cudaStream_t st) {
  if (s.longer) return launch_rows<quantize_i8_long_kernel<kType, kGated, kVec>>(s, st, a);
  if (s.warp) {
    if (s.pieces == 1) return launch_rows<quantize_i8_kernel<1, kType, kGated, kVec, true, false>>(s, st, a);
    return s.pieces == 2 ? launch_rows<quantize_i8_kernel<2, kType, kGated, kVec, true, false>>(s, st, a) : launch_rows<quantize_i8_kernel<4, kType, kGated, kVec, true, false>>(s, st, a);
  }
  if constexpr (kVec) {
    if constexpr (!kGated) {
      if (s.slots && s.pieces == 8) return launch_rows<quantize_i8_kernel<8, kType, kGated, true, false, true>>(s, st, a);
    }
    if (s.slots) return launch_rows<quantize_i8_kernel<4, kType, kGated, true, false, true>>(s, st, a);
  } else if (s.pieces == 8) {
    return launch_rows<quantize_i8_kernel<8, kType, kGated, false, false, false>>(s, st, a);
  }
  if (s.pieces == 1) return launch_rows<quantize_i8_kernel<1, kType, kGated, kVec, false, false>>(s, st, a);
  if (s.pieces == 2) return launch_rows<quantize_i8_kernel<2, kType, kGated, kVec, false, false>>(s, st, a);
  return launch_rows<quantize_i8_kernel<4, kType, kGated, kVec, false, false>>(s, st, a);
}
template <int kType, bool kGated>
static cudaError_t launch_quantize(const QuantI8Args& a, const RowShape& s, bool vec, cudaStream_t st) {
  return vec ? launch_quantize_as<kType, kGated, true>(a, s, st) : launch_quantize_as<kType, kGated, false>(a, s, st);
}
template <int kAll, bool kVec>
static cudaError_t launch_norm_as(const stb_norm& a, const RowShape& s, bool roomy, cudaStream_t st) {
  if (s.warp) {
    if (s.pieces == 1) return launch_rows<block_norm_kernel<kAll, 1, kVec, true, false>>(s, st, a);
    return s.pieces == 2 ? launch_rows<block_norm_kernel<kAll, 2, kVec, true, false>>(s, st, a) : launch_rows<block_norm_kernel<kAll, 4, kVec, true, false>>(s, st, a);
  }
  if constexpr (kVec) {
    if (s.slots && s.pieces == 8) return launch_rows<block_norm_kernel<kAll, 8, true, false, true>>(s, st, a);
    if constexpr (kAll != kAnyType) {
      if (s.slots && !roomy) return launch_rows<block_norm_kernel<kAll, 4, true, false, true>>(s, st, a);
    }
    if (s.slots) return launch_rows<block_norm_kernel<kAll, 4, true, false, true, true>>(s, st, a);
  }
  if (s.pieces == 1) return launch_rows<block_norm_kernel<kAll, 1, kVec, false, false>>(s, st, a);
  if (s.pieces == 2) return launch_rows<block_norm_kernel<kAll, 2, kVec, false, false>>(s, st, a);
  return launch_rows<block_norm_kernel<kAll, kVec ? 4 : 8, kVec, false, false>>(s, st, a);
}
template <int kAll>
static cudaError_t launch_norm(const stb_norm& a, const RowShape& s, bool vec, bool roomy, cudaStream_t st) {
  return vec ? launch_norm_as<kAll, true>(a, s, roomy, st) : launch_norm_as<kAll, false>(a, s, roomy, st);
}
// Whether the norms of rows on their way take 80 registers a thread (nothing is then spilled, of mixed types 12 bytes) or 64 (more rows at a time).  Tokens of mixed types:
// always (2048 x 4096 with an fp32 residual 16.3 us against 19.0; 11008, layer norm with fp32 weights, 45 against 56; 16384 loses, 77 against 70, which is not worth another set
// of kernels; beyond 24576 values eight pieces a thread spill 280 bytes either way).  Of one type: where
// more than three quarters as many threads fit an SM (2048 x 2816 8.1 us against 9.5, 22016 57.9 against 60.1, but 5120 14.2 against 13.0), or, with the norm
// before the gate, as many as that (8192 27.6 against 28.2).
static bool norm_roomy(int h, bool same, bool post) {
  const int threads = ((h + 4 * kPiece - 1) / (4 * kPiece) + 31) / 32 * 32, most = threads <= 512 ? 1024 / threads * threads : 0, roomy = threads <= 768 ? 768 / threads * threads : 0;
  return !same || 4 * roomy > 3 * most || (post && 4 * roomy == 3 * most);
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
  const bool vec = m % stb::kPiece == 0 && stb::rows_aligned(x, ldx, bytes, 8 * bytes) && stb::rows_aligned(x2, ldx2, bytes, 16) && stb::rows_aligned(q, ldq, 1, 8);
  const stb::QuantI8Args a = {x, x2, rows, m, ldx, ldx2, ldq, q, scale};
  const stb::RowShape s = stb::row_shape(m, rows, vec, {xdt == STB_F32 || x2 ? 32u : 16u, 4u * 128u, 1024, x2 ? 0 : (xdt == STB_F32 ? 512 : 1024), x2 ? 1024 : 512, 4});
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool half = xdt == STB_F16;
  const cudaError_t e = x2 ? (half ? stb::launch_quantize<STB_F16, true>(a, s, vec, st) : stb::launch_quantize<STB_BF16, true>(a, s, vec, st))
                           : (xdt == STB_F32 ? stb::launch_quantize<STB_F32, false>(a, s, vec, st)
                                             : (half ? stb::launch_quantize<STB_F16, false>(a, s, vec, st) : stb::launch_quantize<STB_BF16, false>(a, s, vec, st)));
  return e == cudaSuccess ? STB_OK : STB_ERR_CUDA;
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
  const bool vec = a.h % stb::kPiece == 0 && stb::rows_aligned(a.x, a.ldx, xb, 8 * xb) && stb::rows_aligned(a.resid, a.ldr, rb, 8 * rb) && stb::rows_aligned(a.resid_out, a.ldro, rb, 8 * rb) &&
                   stb::rows_aligned(a.y, a.ldy, yb, 8 * yb) && stb::rows_aligned(a.q, a.ldq, 1, 8) && stb::rows_aligned(a.gate, a.tokens > a.tokens_per_gate ? a.ldgate : 0, wb, 8 * wb) &&
                   stb::rows_aligned(a.post_weight, 0, wb, 8 * wb) && stb::rows_aligned(a.post_bias, 0, wb, 8 * wb) && stb::rows_aligned(a.weight, 0, wb, 8 * wb) &&
                   stb::rows_aligned(a.bias, 0, wb, 8 * wb);
  const bool same = a.xdt != STB_F32 && (!residual || a.rdt == a.xdt) && (!vectors || a.wdt == a.xdt);
  const uint32_t each = (a.xdt == STB_F32 ? 32u : 16u) + (!a.resid ? 0u : (a.rdt == STB_F32 ? 32u : 16u));
  const bool roomy = stb::norm_roomy(a.h, same, a.post != 0);
  const stb::RowShape s = stb::row_shape(a.h, a.tokens, vec, {each, 10u * 128u, roomy ? 768 : 1024, 512, roomy ? 768 : 512, 2});
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const cudaError_t e = !same ? stb::launch_norm<stb::kAnyType>(a, s, vec, roomy, st) : (a.xdt == STB_F16 ? stb::launch_norm<STB_F16>(a, s, vec, roomy, st) : stb::launch_norm<STB_BF16>(a, s, vec, roomy, st));
  return e == cudaSuccess ? STB_OK : STB_ERR_CUDA;
}
