// AdamW over many tensors: states in float32, or in 8 bits with a power of two per block of 256.
#include "ops.h"
#include <math.h>

// Every product and sum is rounded by itself, in the order that the header writes them: the 8 bits of a state are those of this arithmetic.
#pragma clang fp contract(off)

using namespace osscar;

namespace {

constexpr int BLOCK = OSSCAR_ADAMW_BLOCK;
static_assert(BLOCK == 256, "32 threads of eight elements");
constexpr int T = 256, CHUNK = T * 8;      // elements of a workgroup
constexpr int TABLE_BYTES = 3860;          // of the kernel's arguments (4096 at most)

// The tensors of a launch, passed by value: nothing has to be copied to the device before, and a captured launch keeps its own.
// NUMBERED: elements are rounded by chance, which goes by their number.
template <bool SMALL, bool MASTER, bool NUMBERED>
struct Table {
  static constexpr int MOST = TABLE_BYTES / (5 * 8 + (NUMBERED ? 8 : 0) + (SMALL ? 16 : 0) + (MASTER ? 8 : 0));
  void* p[MOST];
  const void* g[MOST];
  void* m[MOST];
  void* v[MOST];
  int64_t first[NUMBERED ? MOST : 1];      // number of the tensor's first block in the call
  float* m_scale[SMALL ? MOST : 1];
  float* v_scale[SMALL ? MOST : 1];
  float* master[MASTER ? MOST : 1];
  uint32_t n[MOST];                  // (at most 2^30)
  uint32_t begin[MOST];              // its first workgroup
  int count;
};
struct Step {
  double lr, b1, b2, wd;
  float eps;
  int64_t t;
  const float *lr_dev, *scale_dev;
  const int64_t* t_dev;
  uint32_t seed;
  int random;
};
struct Factors { float b1, c1, b2, c2, decay, step, root; };      // m = b1 m + c1 g, v = b2 v + c2 g g, p = decay p - step (m / (root sqrt(v) + eps))

__host__ __device__ inline double power(double b, int64_t t) {      // (by squaring: the same on both sides)
  double x = 1;
  for (; t > 0; t >>= 1, b *= b)
    if (t & 1) x *= b;
  return x;
}
__host__ __device__ inline Factors factors_of(const Step& s, double lr, int64_t t) {
  return Factors{(float)s.b1, (float)(1 - s.b1), (float)s.b2, (float)(1 - s.b2), (float)(1 - lr * s.wd), (float)(lr / (1 - power(s.b1, t))),
                 (float)(1 / sqrt(1 - power(s.b2, t)))};
}

// A hash of 32 bits: two multiplications by odd numbers (of the golden section and of e), each behind a shift that brings high bits down.
__device__ __forceinline__ uint32_t mix(uint32_t x) {
  x = (x ^ x >> 16) * 0x9E3779B9u;
  x = (x ^ x >> 15) * 0xB7E15163u;
  return x ^ x >> 16;
}
// The bits of z > 0 without its last BITS: to the nearest, halves to even, or (RANDOM) up by chance.
template <int BITS, bool RANDOM>
__device__ __forceinline__ uint32_t keep(float z, uint32_t h) {
  const uint32_t u = __float_as_uint(z);
  return (u + (RANDOM ? h : (1u << (BITS - 1)) - 1 + (u >> BITS & 1))) >> BITS;
}
struct Unit { float scale, inverse; };
// The power of two that is 2^BELOW under the largest power of two in `most` >= 0; NaN and zero for what is not finite.
template <int BELOW>
__device__ __forceinline__ Unit unit_of(float most) {
  const int e = __float_as_int(most) >> 23, at = max(e - BELOW, 1);
  return e == 255 ? Unit{NAN, 0.f} : Unit{__int_as_float(at << 23), __int_as_float((254 - at) << 23)};
}
typedef float v2f __attribute__((ext_vector_type(2)));
// m: sign, four bits of exponent, three of mantissa (the 8-bit float e4m3, which the machine converts), 256 at most.  Rounded by chance: below 2^-6 a sum with it has the step of its smallest
// normal numbers.
template <bool RANDOM>
__device__ __forceinline__ uint32_t codes_m(const float (&y)[4], const uint32_t* h) {
  if constexpr (RANDOM) {
    uint32_t c[4];
#pragma unroll
    for (int e = 0; e < 4; e++) {
      const bool low = fabsf(y[e]) < 0x1p-6f;
      const uint32_t k = keep<20, true>(fabsf(y[e]) + (low ? 0x1p-6f : 0.f), h[e] & 0xFFFFF) - (low ? 121 * 8 : 120 * 8);
      c[e] = k | (__float_as_uint(y[e]) >> 24 & 128);
    }
    return c[0] | c[1] << 8 | c[2] << 16 | c[3] << 24;
  } else {
    int c = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], c, true);
  }
}
__device__ __forceinline__ void values_m(uint32_t c, float (&m)[4]) {
  const v2f a = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, true);
  m[0] = a[0];
  m[1] = a[1];
  m[2] = b[0];
  m[3] = b[1];
}
// sqrt v: four bits of exponent, four of mantissa, whole numbers below 32; what is above zero stays there, so that no m is divided by a lost v.
template <bool RANDOM>
__device__ __forceinline__ uint32_t codes_root(const float (&y)[4], const float (&root)[4], const uint32_t* h) {
  uint32_t c[4];
#pragma unroll
  for (int e = 0; e < 4; e++) {
    const bool low = y[e] < 16.f;
    c[e] = keep<19, RANDOM>(y[e] + (low ? 16.f : 0.f), RANDOM ? (h[e] * 0x9E3779B9u) >> 13 : 0u) - (low ? 131 * 16 : 130 * 16);
    c[e] = max(c[e], root[e] > 0.f ? 1u : 0u);
  }
  return c[0] | c[1] << 8 | c[2] << 16 | c[3] << 24;
}
__device__ __forceinline__ void values_root(uint32_t c, float (&r)[4]) {
#pragma unroll
  for (int e = 0; e < 4; e++) {
    const uint32_t k = c >> (8 * e) & 255;
    const bool low = k < 16;
    r[e] = __uint_as_float((k + (low ? 131 * 16 : 130 * 16)) << 19) - (low ? 16.f : 0.f);
  }
}

__device__ __forceinline__ float largest_of_32(float x) {      // NaN where one is: the largest of the bits of what is not negative
  uint32_t u = __float_as_uint(x);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) { const uint32_t w = __shfl_xor(u, o, 32); u = w > u ? w : u; }
  return __uint_as_float(u);
}
// Eight codes, four in a word
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef u32x2 u32x2_any __attribute__((aligned(1)));
__device__ __forceinline__ u32x2 load_codes(const void* p, int64_t at, int64_t most) {
  const uint8_t* q = reinterpret_cast<const uint8_t*>(p) + at;
  if (most >= 8) return *reinterpret_cast<const u32x2_any*>(q);
  u32x2 w{0, 0};
#pragma unroll
  for (int e = 0; e < 8; e++) if (e < most) w[e / 4] |= (uint32_t)q[e] << (8 * (e % 4));
  return w;
}
__device__ __forceinline__ void store_codes(void* p, int64_t at, const u32x2& w, int64_t most) {
  uint8_t* q = reinterpret_cast<uint8_t*>(p) + at;
  if (most >= 8) { *reinterpret_cast<u32x2_any*>(q) = w; return; }
#pragma unroll
  for (int e = 0; e < 8; e++) if (e < most) q[e] = (uint8_t)(w[e / 4] >> (8 * (e % 4)));
}
template <class F>
__device__ __forceinline__ void in_fours(F f) { f(0); f(1); }

// The tensor of this workgroup: how many of them begin at or before it.
template <class Tab>
__device__ __forceinline__ int tensor_of(const Tab& t, uint32_t block) {
  int i = 0;
  for (int base = 0; base < t.count; base += 64) {
    const int k = base + (threadIdx.x & 63);
    i += __popcll(__ballot(k < t.count && t.begin[k < t.count ? k : 0] <= block));
  }
  return __builtin_amdgcn_readfirstlane(i - 1);
}

// One pass over a chunk of one tensor, eight elements a thread.  Bound by reading and writing parameters and states: 50 M of bf16 with a float32 copy 262 us (5.4 TB/s), 4.9 M of float32 in 192
// tensors 28 us.  In 8 bits the vector units are as busy: 308 M of bf16, by chance, 750 us (4.1 TB/s), 22 M of float32, to the nearest, 61 us (5.9).
template <bool P32, bool G32, bool MASTER, bool SMALL, bool RANDOM>
__global__ __launch_bounds__(T) void adamw_kernel(const Table<SMALL, MASTER, RANDOM> tab, const Step s, Factors f) {
  constexpr bool CODED_P = RANDOM && !P32 && !MASTER;      // bf16 parameters rounded by chance
  const int i = tensor_of(tab, blockIdx.x);
  const int64_t n = tab.n[i], at = (int64_t)(blockIdx.x - tab.begin[i]) * CHUNK + threadIdx.x * 8, most = n - at;
  const bool mine = most > 0;
  typedef Eight<P32 || MASTER> EP;
  typedef Eight<G32> EG;
  typename EP::type rp{};
  typename EG::type rg{};
  typename Eight<true>::type rm{}, rv{};
  u32x2 cm{0, 0}, cv{0, 0};
  float ms = 0.f, vs = 0.f;
  void* kept;
  if constexpr (MASTER) kept = tab.master[i];
  else kept = tab.p[i];
  const void* grad = tab.g[i];
  void *am = tab.m[i], *av = tab.v[i];
  auto fetch = [&](int64_t all) {
    rp = EP::load(kept, at, all);
    rg = EG::load(grad, at, all);
    if constexpr (SMALL) {
      cm = load_codes(am, at, all);
      cv = load_codes(av, at, all);
      ms = tab.m_scale[i][at / BLOCK];
      vs = tab.v_scale[i][at / BLOCK];
    } else {
      rm = Eight<true>::load(am, at, all);
      rv = Eight<true>::load(av, at, all);
    }
  };
  if (most >= 8) fetch(8);
  else if (mine) fetch(most);
  const int64_t t = s.t_dev ? max(*s.t_dev, (int64_t)1) : s.t;
  if (s.t_dev || s.lr_dev) f = factors_of(s, s.lr_dev ? (double)*s.lr_dev : s.lr, t);
  float gs = 1.f;
  if (s.scale_dev) {
    gs = *s.scale_dev;
    if (!(fabsf(gs) < INFINITY)) return;      // the step is left out
  }
  float p[8], g[8], m[8], v[8], root[8];
  EP::values(rp, p);
  EG::values(rg, g);
  if constexpr (SMALL) {
    in_fours([&](int k) {
      float x[4], r[4];
      values_m(cm[k], x);
      values_root(cv[k], r);
#pragma unroll
      for (int e = 0; e < 4; e++) {
        m[4 * k + e] = x[e] * ms;
        r[e] *= vs;
        v[4 * k + e] = r[e] * r[e];
      }
    });
  } else {
    Eight<true>::values(rm, m);
    Eight<true>::values(rv, v);
  }
#pragma unroll
  for (int e = 0; e < 8; e++) {
    if (s.scale_dev) g[e] = g[e] * gs;
    m[e] = m[e] * f.b1 + g[e] * f.c1;
    v[e] = v[e] * f.b2 + (g[e] * g[e]) * f.c2;
    root[e] = sqrtf(v[e]);
    p[e] = p[e] * f.decay - f.step * (m[e] / (root[e] * f.root + s.eps));
  }
  uint32_t h[8] = {};
  if constexpr (SMALL ? RANDOM : CODED_P) {
    const uint64_t number = (uint64_t)tab.first[i] * BLOCK + (uint64_t)at;      // of the element in the call; eight of them have one high half
    const uint32_t key = mix((uint32_t)(number >> 32) ^ mix(s.seed + (s.t_dev ? (uint32_t)t : 0u)));
#pragma unroll
    for (int e = 0; e < 8; e++) h[e] = mix(((uint32_t)number + e) ^ key);
  }
  Unit um, ur;
  if constexpr (SMALL) {
    uint32_t mm = 0, mr = 0;
#pragma unroll
    for (int e = 0; e < 8; e++) {      // (as bits, so that a NaN is the largest; what is past the end is zero, as its gradient was)
      mm = max(mm, __float_as_uint(m[e]) & 0x7FFFFFFFu);
      mr = max(mr, __float_as_uint(root[e]) & 0x7FFFFFFFu);
    }
    um = unit_of<7>(largest_of_32(__uint_as_float(mm)));
    ur = unit_of<17>(largest_of_32(__uint_as_float(mr)));
    in_fours([&](int k) {
      float y[4], z[4], r[4];
#pragma unroll
      for (int e = 0; e < 4; e++) {
        y[e] = m[4 * k + e] * um.inverse;
        r[e] = root[4 * k + e];
        z[e] = r[e] * ur.inverse;
      }
      cm[k] = um.inverse > 0.f ? codes_m<RANDOM>(y, h + 4 * k) : 0u;
      cv[k] = ur.inverse > 0.f ? codes_root<RANDOM>(z, r, h + 4 * k) : 0u;
    });
  }
  auto store = [&](int64_t all) {
    if constexpr (CODED_P) {      // up by chance, as its part of a step is
      u16x8 w;
#pragma unroll
      for (int e = 0; e < 8; e++) w[e] = fabsf(p[e]) < INFINITY ? (uint16_t)((__float_as_uint(p[e]) + (h[e] >> 16)) >> 16) : bf16_nearest(p[e]);
      uint16_t* q = reinterpret_cast<uint16_t*>(kept) + at;
      if (all >= 8) *reinterpret_cast<u16x8_any*>(q) = w;
      else {
#pragma unroll
        for (int e = 0; e < 8; e++) if (e < all) q[e] = w[e];
      }
    } else {
      EP::store(kept, at, p, all);
    }
    if constexpr (MASTER) Eight<false>::store(tab.p[i], at, p, all);
    if constexpr (SMALL) {
      store_codes(am, at, cm, all);
      store_codes(av, at, cv, all);
      if ((threadIdx.x & 31) == 0) {
        tab.m_scale[i][at / BLOCK] = um.scale;
        tab.v_scale[i][at / BLOCK] = ur.scale;
      }
    } else {
      Eight<true>::store(am, at, m, all);
      Eight<true>::store(av, at, v, all);
    }
  };
  if (most >= 8) store(8);
  else if (mine) store(most);
}

// What 8-bit states stand for, in bf16, which holds them exactly but for m of scales below 2^-124 (3 bits above steps of 2^-135): 308 M 334 us, 5.5 TB/s.
struct Values {
  static constexpr int MOST = TABLE_BYTES / (7 * 8 + 4);
  const void *m[MOST], *v[MOST];
  const float *m_scale[MOST], *v_scale[MOST];
  uint16_t *m_out[MOST], *root_out[MOST];
  int64_t n[MOST];
  uint32_t begin[MOST];
  int count;
};
__global__ __launch_bounds__(T) void values_kernel(const Values tab) {
  const int i = tensor_of(tab, blockIdx.x);
  const int64_t n = tab.n[i], at = (int64_t)(blockIdx.x - tab.begin[i]) * CHUNK + threadIdx.x * 8, most = n - at;
  if (most <= 0) return;
  const u32x2 cm = load_codes(tab.m[i], at, most), cv = load_codes(tab.v[i], at, most);
  const float ms = tab.m_scale[i][at / BLOCK], vs = tab.v_scale[i][at / BLOCK];
  float m[8], r[8];
  in_fours([&](int k) {
    float x[4], y[4];
    values_m(cm[k], x);
    values_root(cv[k], y);
#pragma unroll
    for (int e = 0; e < 4; e++) {
      m[4 * k + e] = x[e] * ms;
      r[4 * k + e] = y[e] * vs;
    }
  });
  Eight<false>::store(tab.m_out[i], at, m, most);
  Eight<false>::store(tab.root_out[i], at, r, most);
}

constexpr int64_t LAUNCH = 1 << 23;      // workgroups of a launch (HIP cuts 2^32 threads off)

// Goes over the tensors of one kind, launch by launch: fill(table, place in it, tensor, elements before this launch's part of it).
template <class Tab, class Fill, class Go>
void in_launches(int64_t count, const osscar_adamw_tensor* t, bool (*kind)(const osscar_adamw_tensor&, int), int which, Fill fill, Go go) {
  Tab tab;
  int64_t blocks = 0;
  tab.count = 0;
  auto flush = [&] {
    if (tab.count > 0) go(tab, (unsigned)blocks);
    tab.count = 0;
    blocks = 0;
  };
  int64_t first = 0;
  for (int64_t k = 0; k < count; k++) {
    const int64_t number = first;
    first += (t[k].n + BLOCK - 1) / BLOCK;
    if (t[k].n == 0 || !kind(t[k], which)) continue;
    const int64_t need = (t[k].n + CHUNK - 1) / CHUNK;      // (n is at most 2^30: 2^19 workgroups)
    if (tab.count == Tab::MOST || blocks + need > LAUNCH) flush();
    fill(tab, tab.count, t[k], number);
    tab.begin[tab.count] = (uint32_t)blocks;
    tab.count++;
    blocks += need;
  }
  flush();
}

int kind_of(const osscar_adamw_tensor& t) { return (t.master ? 2 : t.p_dtype == OSSCAR_F32 ? 0 : 1) * 2 + (t.g_dtype == OSSCAR_F32 ? 1 : 0); }
bool is_kind(const osscar_adamw_tensor& t, int which) { return kind_of(t) == which; }
bool any_kind(const osscar_adamw_tensor&, int) { return true; }

template <bool P32, bool G32, bool MASTER, bool SMALL, bool RANDOM>
void steps(const osscar_adamw_tensor* t, int64_t count, const Step& s, const Factors& f, hipStream_t stream) {
  if constexpr (RANDOM && !SMALL && (P32 || MASTER)) {      // (nothing is rounded to fewer bits but copies of masters)
    steps<P32, G32, MASTER, SMALL, false>(t, count, s, f, stream);
  } else {
    typedef Table<SMALL, MASTER, RANDOM> Tab;
    static_assert(sizeof(Tab) + sizeof(Step) + sizeof(Factors) <= 4096, "a launch's arguments");
    in_launches<Tab>(
        count, t, is_kind, (MASTER ? 2 : P32 ? 0 : 1) * 2 + (G32 ? 1 : 0),
        [](Tab& tab, int at, const osscar_adamw_tensor& x, int64_t number) {
          tab.p[at] = x.p;
          tab.g[at] = x.g;
          tab.m[at] = x.m;
          tab.v[at] = x.v;
          tab.n[at] = (uint32_t)x.n;
          if constexpr (RANDOM) tab.first[at] = number;
          if constexpr (SMALL) { tab.m_scale[at] = x.m_scale; tab.v_scale[at] = x.v_scale; }
          if constexpr (MASTER) tab.master[at] = x.master;
        },
        [&](const Tab& tab, unsigned blocks) { hipLaunchKernelGGL((adamw_kernel<P32, G32, MASTER, SMALL, RANDOM>), dim3(blocks), dim3(T), 0, stream, tab, s, f); });
  }
}
template <bool SMALL, bool RANDOM>
void steps_of(const osscar_adamw_tensor* t, int64_t count, const Step& s, const Factors& f, hipStream_t stream) {
  bool seen[6] = {};
  for (int64_t k = 0; k < count; k++)
    if (t[k].n > 0) seen[kind_of(t[k])] = true;
  if (seen[0]) steps<true, false, false, SMALL, RANDOM>(t, count, s, f, stream);
  if (seen[1]) steps<true, true, false, SMALL, RANDOM>(t, count, s, f, stream);
  if (seen[2]) steps<false, false, false, SMALL, RANDOM>(t, count, s, f, stream);
  if (seen[3]) steps<false, true, false, SMALL, RANDOM>(t, count, s, f, stream);
  if (seen[4]) steps<false, false, true, SMALL, RANDOM>(t, count, s, f, stream);
  if (seen[5]) steps<false, true, true, SMALL, RANDOM>(t, count, s, f, stream);
}

const char* bad_tensor(const osscar_adamw_tensor& t, bool small, bool values) {
  if (!a_size(t.n, 0)) return "osscar_adamw: a tensor's size is negative or above 2^30";
  if (t.n == 0) return nullptr;
  if (!t.m || !t.v) return "osscar_adamw: NULL pointer";
  if (small ? !t.m_scale || !t.v_scale || (((uintptr_t)t.m_scale | (uintptr_t)t.v_scale) & 3) : (((uintptr_t)t.m | (uintptr_t)t.v) & 3) != 0)
    return "osscar_adamw: a state is missing or not aligned to its elements";
  if (values) return nullptr;
  if (!real_dtype(t.p_dtype) || !real_dtype(t.g_dtype)) return "osscar_adamw: unknown dtype";
  if (!t.p || !t.g) return "osscar_adamw: NULL pointer";
  if (t.master && t.p_dtype != OSSCAR_BF16) return "osscar_adamw: a float32 copy goes with bf16 parameters";
  if (((uintptr_t)t.p & (t.p_dtype == OSSCAR_F32 ? 3 : 1)) || ((uintptr_t)t.g & (t.g_dtype == OSSCAR_F32 ? 3 : 1)) || ((uintptr_t)t.master & 3))
    return "osscar_adamw: a buffer is not aligned to its elements";
  return nullptr;
}

}  // namespace

extern "C" osscar_status osscar_adamw(const osscar_adamw_tensor* tensors, int64_t count, const osscar_adamw_desc* d, void* hip_stream) {
  const char* bad = nullptr;
  if (!d || count < 0 || count > (int64_t)1 << 30 || (count > 0 && !tensors)) bad = "osscar_adamw: NULL pointer or negative count";
  if (!bad && d->bits != 8 && d->bits != 32) bad = "osscar_adamw: states have 8 or 32 bits";
  // (written so that NaN is refused)
  if (!bad && !(d->beta1 >= 0 && d->beta1 < 1 && d->beta2 >= 0 && d->beta2 < 1)) bad = "osscar_adamw: beta1 and beta2 are at least 0 and below 1";
  if (!bad && !((float)d->eps > 0.f && (float)d->eps < INFINITY)) bad = "osscar_adamw: eps must be a positive float32";
  if (!bad && !(d->weight_decay >= 0 && d->weight_decay < INFINITY)) bad = "osscar_adamw: weight_decay must not be negative";
  if (!bad && !d->lr_dev && !(d->lr >= 0 && (float)d->lr < INFINITY)) bad = "osscar_adamw: lr must not be negative";
  if (!bad && !d->step_dev && d->step < 1) bad = "osscar_adamw: steps count from 1";
  if (!bad && (((uintptr_t)d->lr_dev & 3) || ((uintptr_t)d->step_dev & 7) || ((uintptr_t)d->grad_scale_dev & 3))) bad = "osscar_adamw: a buffer is not aligned to its elements";
  bool any = false;
  for (int64_t k = 0; !bad && k < count; k++) { bad = bad_tensor(tensors[k], d->bits == 8, false); any = any || tensors[k].n > 0; }
  if (bad) return refuse_call(OSSCAR_EINVAL, bad);
  if (!any) return OSSCAR_OK;
  const Step s{d->lr, d->beta1, d->beta2, d->weight_decay, (float)d->eps, d->step, d->lr_dev, d->grad_scale_dev, d->step_dev, d->seed, d->stochastic != 0};
  const Factors f = factors_of(s, d->lr_dev ? 0 : d->lr, d->step_dev ? 1 : d->step);
  hipStream_t stream = reinterpret_cast<hipStream_t>(hip_stream);
  if (d->bits == 8 && s.random) steps_of<true, true>(tensors, count, s, f, stream);
  else if (d->bits == 8) steps_of<true, false>(tensors, count, s, f, stream);
  else if (s.random) steps_of<false, true>(tensors, count, s, f, stream);
  else steps_of<false, false>(tensors, count, s, f, stream);
  return launched();
}

extern "C" osscar_status osscar_adamw_values(const osscar_adamw_tensor* tensors, int64_t count, void* const* m_out, void* const* root_out, void* hip_stream) {
  const char* bad = nullptr;
  bool any = false;
  if (count < 0 || count > (int64_t)1 << 30 || (count > 0 && (!tensors || !m_out || !root_out))) bad = "osscar_adamw_values: NULL pointer or negative count";
  for (int64_t k = 0; !bad && k < count; k++) {
    bad = bad_tensor(tensors[k], true, true);
    if (!bad && tensors[k].n > 0 && (!m_out[k] || !root_out[k] || (((uintptr_t)m_out[k] | (uintptr_t)root_out[k]) & 1))) bad = "osscar_adamw_values: an output is missing or not aligned to its elements";
    any = any || tensors[k].n > 0;
  }
  if (bad) return refuse_call(OSSCAR_EINVAL, bad);
  if (!any) return OSSCAR_OK;
  hipStream_t stream = reinterpret_cast<hipStream_t>(hip_stream);
  static_assert(sizeof(Values) <= 4096, "a launch's arguments");
  in_launches<Values>(
      count, tensors, any_kind, 0,
      [&](Values& tab, int at, const osscar_adamw_tensor& x, int64_t) {
        const int64_t k = &x - tensors;
        tab.m[at] = x.m;
        tab.v[at] = x.v;
        tab.m_scale[at] = x.m_scale;
        tab.v_scale[at] = x.v_scale;
        tab.m_out[at] = reinterpret_cast<uint16_t*>(m_out[k]);
        tab.root_out[at] = reinterpret_cast<uint16_t*>(root_out[k]);
        tab.n[at] = x.n;
      },
      [&](const Values& tab, unsigned blocks) { hipLaunchKernelGGL(values_kernel, dim3(blocks), dim3(T), 0, stream, tab); });
  return launched();
}
