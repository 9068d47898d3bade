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

// Eight neighbouring elements of a row as they are in memory, so that few registers hold what is under way; zeros from the `most`-th on.
template <bool F32> struct Eight;
template <> struct Eight<false> {
  typedef u16x8 type;
  static __device__ __forceinline__ type load(const void* p, int64_t at, int64_t most = 8) {
    const uint16_t* q = reinterpret_cast<const uint16_t*>(p) + at;
    if (most >= 8) return *reinterpret_cast<const u16x8_any*>(q);
    type w;
#pragma unroll
    for (int e = 0; e < 8; e++) { w[e] = 0; if (e < most) w[e] = q[e]; }
    return w;
  }
  static __device__ __forceinline__ void values(const type& w, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 8; e++) v[e] = bf16_value(w[e]);
  }
  static __device__ __forceinline__ void store(void* p, int64_t at, const float (&v)[8], int64_t most = 8) {
    uint16_t* q = reinterpret_cast<uint16_t*>(p) + at;
    u16x8 w;
#pragma unroll
    for (int e = 0; e < 8; e++) w[e] = bf16_nearest(v[e]);
    if (most >= 8) { *reinterpret_cast<u16x8_any*>(q) = w; return; }
#pragma unroll
    for (int e = 0; e < 8; e++) if (e < most) q[e] = w[e];
  }
};
template <> struct Eight<true> {
  struct type { f32x4 a, b; };
  static __device__ __forceinline__ type load(const void* p, int64_t at, int64_t most = 8) {
    const float* q = reinterpret_cast<const float*>(p) + at;
    if (most >= 8) return type{*reinterpret_cast<const f32x4_any*>(q), *reinterpret_cast<const f32x4_any*>(q + 4)};
    type w;
#pragma unroll
    for (int e = 0; e < 4; e++) {
      w.a[e] = w.b[e] = 0.f;
      if (e < most) w.a[e] = q[e];
      if (e + 4 < most) w.b[e] = q[e + 4];
    }
    return w;
  }
  static __device__ __forceinline__ void values(const type& w, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 4; e++) { v[e] = w.a[e]; v[e + 4] = w.b[e]; }
  }
  static __device__ __forceinline__ void store(void* p, int64_t at, const float (&v)[8], int64_t most = 8) {
    float* q = reinterpret_cast<float*>(p) + at;
    if (most >= 8) {
      *reinterpret_cast<f32x4_any*>(q) = f32x4{v[0], v[1], v[2], v[3]};
      *reinterpret_cast<f32x4_any*>(q + 4) = f32x4{v[4], v[5], v[6], v[7]};
      return;
    }
#pragma unroll
    for (int e = 0; e < 8; e++) if (e < most) q[e] = v[e];
  }
};

// Eight elements of a row from its c-th, in the wave that the row ends in, without a branch for each of them (what is past the end is anything): bf16 from eight before the end on and
// moved to their places, float32 (where that is 24 moves) one by one, the last one again past the end.  A row of fewer than eight bf16 is read one by one.
template <bool F32>
__device__ __forceinline__ typename Eight<F32>::type edge_load(const void* p, int64_t row_at, int c, int C) {
  if constexpr (F32) {
    const float* q = reinterpret_cast<const float*>(p) + row_at;
    typename Eight<true>::type w;
#pragma unroll
    for (int e = 0; e < 4; e++) {
      w.a[e] = q[min(c + e, C - 1)];
      w.b[e] = q[min(c + e + 4, C - 1)];
    }
    return w;
  } else {
    if (C < 8) return Eight<false>::load(p, row_at + c, C - c);
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    const int at = min(c, C - 8), s = c - at;
    u32x4 x = __builtin_bit_cast(u32x4, Eight<false>::load(p, row_at + at));
    if (s & 4) x = u32x4{x[2], x[3], x[3], x[3]};
    if (s & 2) x = u32x4{x[1], x[2], x[3], x[3]};
    if (s & 1) x = u32x4{x[0] >> 16 | x[1] << 16, x[1] >> 16 | x[2] << 16, x[2] >> 16 | x[3] << 16, x[3] >> 16};
    return __builtin_bit_cast(u16x8, x);
  }
}

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
