// What the operators without a context share: refusals, the carving of the caller's workspace, bf16.
#pragma once
#include "../../include/osscar.h"
#include "internal.h"

namespace osscar {

inline osscar_status refuse_call(osscar_status st, const char* msg) { set_contextless_error(msg); return st; }
inline osscar_status launched() {
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) return OSSCAR_OK;
  return refuse_call(OSSCAR_EHIP, hipGetErrorString(e));
}
inline bool real_dtype(int32_t t) { return t == OSSCAR_F32 || t == OSSCAR_BF16; }
// HIP cuts launches of 2^32 threads along a dimension off, without an error.
inline bool launchable(int64_t blocks, int64_t threads) { return blocks * threads < (int64_t)1 << 32; }
inline bool a_size(int64_t v, int64_t low) { return v >= low && v <= (int64_t)1 << 30; }

// Pieces of a workspace, each at a 256-byte boundary.  With base = nullptr it only counts.
struct Carve {
  char* base; size_t used = 0;
  explicit Carve(void* p) : base(reinterpret_cast<char*>(p)) {}
  char* take(size_t bytes) {
    char* p = base ? base + used : nullptr;
    used += (bytes + 255) / 256 * 256;
    return p;
  }
};

__device__ __forceinline__ float bf16_value(uint16_t b) { return __uint_as_float((uint32_t)b << 16); }
__device__ __forceinline__ uint16_t bf16_nearest(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }

// Vectors at any alignment that their elements have.
typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
typedef u16x8 u16x8_any __attribute__((aligned(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef f32x4 f32x4_any __attribute__((aligned(4)));

// C neighbouring values of a row, of which the ones before `most` exist
template <int C>
__device__ __forceinline__ void put_bf16(uint16_t* p, const float (&v)[C], int most) {
  static_assert(C % 8 == 0, "");
  if (most >= C) {
#pragma unroll
    for (int c = 0; c < C; c += 8) {
      u16x8 w;
#pragma unroll
      for (int e = 0; e < 8; e++) w[e] = bf16_nearest(v[c + e]);
      *reinterpret_cast<u16x8_any*>(p + c) = w;
    }
  } else {
#pragma unroll
    for (int c = 0; c < C; c++)
      if (c < most) p[c] = bf16_nearest(v[c]);
  }
}
template <int C>
__device__ __forceinline__ void put_f32(float* p, const float (&v)[C], int most) {
  if (most >= C) {
#pragma unroll
    for (int c = 0; c < C; c += 4) *reinterpret_cast<f32x4_any*>(p + c) = f32x4{v[c], v[c + 1], v[c + 2], v[c + 3]};
  } else {
#pragma unroll
    for (int c = 0; c < C; c++)
      if (c < most) p[c] = v[c];
  }
}
template <int C>
__device__ __forceinline__ void get_values(const void* p, int64_t at, int f32, float (&v)[C], int most) {
  if (f32) {
    const float* q = reinterpret_cast<const float*>(p) + at;
    if (most >= C) {
#pragma unroll
      for (int c = 0; c < C; c += 4) {
        const f32x4 w = *reinterpret_cast<const f32x4_any*>(q + c);
#pragma unroll
        for (int e = 0; e < 4; e++) v[c + e] = w[e];
      }
    } else {
#pragma unroll
      for (int c = 0; c < C; c++) v[c] = c < most ? q[c] : 0.f;
    }
  } else {
    const uint16_t* q = reinterpret_cast<const uint16_t*>(p) + at;
    if (most >= C) {
#pragma unroll
      for (int c = 0; c < C; c += 8) {
        const u16x8 w = *reinterpret_cast<const u16x8_any*>(q + c);
#pragma unroll
        for (int e = 0; e < 8; e++) v[c + e] = bf16_value(w[e]);
      }
    } else {
#pragma unroll
      for (int c = 0; c < C; c++) v[c] = c < most ? bf16_value(q[c]) : 0.f;
    }
  }
}

}  // namespace osscar
