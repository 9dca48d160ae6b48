// What the kernels of a decoder layer in few bits share: element types, conversions, matrix-core operands, and the
// reading of a paged cache's description (the struct of include/bmx.h) with every index from device memory checked.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/bmx.h"
#include "kv_range.h"

namespace bmx {

using f32x4 = float __attribute__((ext_vector_type(4)));
using f16x2 = _Float16 __attribute__((ext_vector_type(2)));
using f16x8 = _Float16 __attribute__((ext_vector_type(8)));
using bf16x8 = __bf16 __attribute__((ext_vector_type(8)));
using u32x4 = uint32_t __attribute__((ext_vector_type(4)));
using u32x2 = uint32_t __attribute__((ext_vector_type(2)));

__host__ __device__ static inline int type_bytes(int type) { return type == BMX_F32 ? 4 : 2; }
// Bytes that a token's head takes in a page.
__host__ __device__ static inline int kv_row_bytes(int dim) { return (dim + 31) / 32 * 32; }

__device__ static inline float bf16_float(uint32_t bits) { return __builtin_bit_cast(float, bits << 16); }
// Round to nearest, ties to even (NaN stays NaN).
__device__ static inline uint32_t bf16_bits(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }
__device__ static inline uint32_t f16_bits(float x) { return __builtin_bit_cast(uint16_t, (_Float16)x); }

template <int TYPE>
__device__ static inline float load_one(const void* p, int64_t at) {
  if constexpr (TYPE == BMX_F32) return static_cast<const float*>(p)[at];
  else if constexpr (TYPE == BMX_F16) return (float)static_cast<const _Float16*>(p)[at];
  else return bf16_float(static_cast<const uint16_t*>(p)[at]);
}
template <int TYPE>
__device__ static inline void store_one(void* p, int64_t at, float x) {
  if constexpr (TYPE == BMX_F32) static_cast<float*>(p)[at] = x;
  else if constexpr (TYPE == BMX_F16) static_cast<uint16_t*>(p)[at] = (uint16_t)f16_bits(x);
  else static_cast<uint16_t*>(p)[at] = (uint16_t)bf16_bits(x);
}

// Eight consecutive values as floats, `left` of them there (the others are 0); ALIGNED: the address is 16-byte aligned.
template <int TYPE>
__device__ static inline void load_eight(const void* p, int64_t at, int left, bool aligned, float (&x)[8]) {
  if (left >= 8 && aligned) {
    if constexpr (TYPE == BMX_F32) {
      const f32x4 a = *reinterpret_cast<const f32x4*>(static_cast<const float*>(p) + at);
      const f32x4 b = *reinterpret_cast<const f32x4*>(static_cast<const float*>(p) + at + 4);
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = a[j], x[4 + j] = b[j];
    } else {
      const u32x4 a = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(p) + at);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t h = (a[j / 2] >> (16 * (j % 2))) & 0xffff;
        x[j] = TYPE == BMX_F16 ? (float)__builtin_bit_cast(_Float16, (uint16_t)h) : bf16_float(h);
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = j < left ? load_one<TYPE>(p, at + j) : 0.0f;
  }
}

// N consecutive values, as they lie in memory at an address of an element.
template <int TYPE, int N>
struct Run {
  static constexpr int kDwords = N * (TYPE == BMX_F32 ? 4 : 2) / 4;
  struct __attribute__((packed, aligned(TYPE == BMX_F32 ? 4 : 2))) Raw {
    uint32_t w[kDwords];
  };
  uint32_t w[kDwords];

  __device__ static size_t bytes(int64_t at) { return at * (TYPE == BMX_F32 ? 4 : 2); }
  // `left` of them are there, the others are 0
  __device__ void load(const void* p, int64_t at, int left) {
    if (left >= N) {
      const Raw r = *reinterpret_cast<const Raw*>(static_cast<const char*>(p) + bytes(at));
#pragma unroll
      for (int i = 0; i < kDwords; ++i) w[i] = r.w[i];
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j) {
        if constexpr (TYPE == BMX_F32) {
          w[j] = j < left ? static_cast<const uint32_t*>(p)[at + j] : 0;
        } else {
          const uint32_t h = j < left ? static_cast<const uint16_t*>(p)[at + j] : 0;
          w[j / 2] = j % 2 ? w[j / 2] | h << 16 : h;
        }
      }
    }
  }
  __device__ void store(void* p, int64_t at, int left) const {
    if (left >= N) {
      Raw r;
#pragma unroll
      for (int i = 0; i < kDwords; ++i) r.w[i] = w[i];
      *reinterpret_cast<Raw*>(static_cast<char*>(p) + bytes(at)) = r;
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j) {
        if (j >= left) continue;
        if constexpr (TYPE == BMX_F32) static_cast<uint32_t*>(p)[at + j] = w[j];
        else static_cast<uint16_t*>(p)[at + j] = (uint16_t)(w[j / 2] >> (16 * (j % 2)));
      }
    }
  }
  __device__ float get(int j) const {
    if constexpr (TYPE == BMX_F32) {
      const uint32_t x = w[j];
      return __builtin_bit_cast(float, x);
    } else {
      const uint32_t h = w[j / 2] >> (16 * (j % 2)) & 0xffff;
      return TYPE == BMX_F16 ? (float)__builtin_bit_cast(_Float16, (uint16_t)h) : bf16_float(h);
    }
  }
  __device__ void set2(int j, float a, float b) {  // values j (even) and j + 1
    if constexpr (TYPE == BMX_F32) w[j] = __builtin_bit_cast(uint32_t, a), w[j + 1] = __builtin_bit_cast(uint32_t, b);
    else if constexpr (TYPE == BMX_F16) w[j / 2] = f16_bits(a) | f16_bits(b) << 16;
    else w[j / 2] = bf16_bits(a) | bf16_bits(b) << 16;
  }
};

// A sequence's rows and positions (lengths and starts come from device memory); Cache: bmx_kv_cache or bmx_kv4_cache.
template <class Cache>
__device__ static inline KvSpan kv_span(const Cache& c, int seq, int rows, int max_new) {
  const int each = c.starts ? 0 : rows / c.sequences, begin = c.starts ? c.starts[seq] : seq * each, end = c.starts ? c.starts[seq + 1] : begin + each;
  return kv_span_of(begin, end, c.lengths[seq], rows, max_new, c.table_width);
}
// The page at place `at` of a sequence's row of the table; negative where there is none.
template <class Cache>
__device__ static inline int kv_page(const Cache& c, int seq, int at) {
  const int p = c.table[seq * c.table_ld + at];
  return p < c.num_pages ? p : -1;
}

// Where a page's keys and values of one head hold token t, value d (row: kv_row_bytes).
__device__ static inline int kv_key_at(int row, int t, int d) {
  const int base = t / 16 * 16 * row + d / 64 * 1024;
  return d / 64 * 64 + 64 <= row ? base + d % 64 / 16 * 256 + t % 16 * 16 + d % 16 : base + d % 32 / 8 * 128 + t % 16 * 8 + d % 8;
}
__device__ static inline int kv_value_at(int t, int d) { return d / 16 * 1024 + t % 16 / 4 * 256 + d % 16 * 16 + t / 16 * 4 + t % 4; }
// Bytes that a token's head takes in a page of 4 bits, and where its value d lies there: the low half of a byte if d is even.
__host__ __device__ static inline int kv4_row_bytes(int dim) { return (dim + 31) / 32 * 16; }
__device__ static inline int kv4_key_at(int row, int t, int d) { return t * row + d / 2; }
__device__ static inline int kv4_value_at(int t, int d) { return d / 32 * 1024 + t % 16 / 4 * 256 + d % 32 / 2 * 16 + t / 16 * 4 + t % 4; }

// Memory as a buffer of so many bytes.  A read whose lane_at is behind its end gives zeros and moves nothing; what the hardware compares with the end
// need not hold `at`, so lane_at alone says whether there is anything to read (kNowhere added: there is not).
constexpr int kNowhere = 1 << 30;
using Rsrc = __amdgpu_buffer_rsrc_t;
__device__ inline Rsrc buffer(const void* p, int bytes) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, bytes, 0x00027000); }
// (lane_at differs from lane to lane, at does not)
__device__ inline u32x4 load16(Rsrc r, int lane_at, int at) { return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, lane_at, at, 0)); }
__device__ inline u32x2 load8(Rsrc r, int lane_at, int at) { return __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(r, lane_at, at, 0)); }
__device__ inline uint32_t load4(Rsrc r, int lane_at, int at) { return __builtin_amdgcn_raw_buffer_load_b32(r, lane_at, at, 0); }

// The upper halves of two dwords.
__device__ inline uint32_t upper_halves(float a, float b) {
  return __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, b), __builtin_bit_cast(uint32_t, a), 0x07060302u);
}
// What the upper half of a value leaves.
__device__ inline float lower_part(float a) { return a - __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, a) & 0xffff0000u); }

}  // namespace bmx
