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
constexpr int TABLE_BYTES = 3600;          // of the kernel's arguments (4096 at most)

// The tensors of a launch, passed by value: nothing has to be copied to the device before, and a captured launch keeps its own.
template <bool SMALL, bool MASTER>
struct Table {
  static constexpr int MOST = TABLE_BYTES / (6 * 8 + 4 + (SMALL ? 16 : 0) + (MASTER ? 8 : 0));
  void* p[MOST];
  const void* g[MOST];
  void* m[MOST];
  void* v[MOST];
  int64_t n[MOST];
  int64_t first[MOST];               // number of the tensor's first block in the call
  float* m_scale[SMALL ? MOST : 1];
  float* v_scale[SMALL ? MOST : 1];
  float* master[MASTER ? MOST : 1];
  uint32_t begin[MOST];              // its first workgroup
  int count;
};
struct Step {
  double lr, b1, b2, wd;
  float eps, grad_scale;
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
// The bits of z > 0 without its last BITS: to the nearest, halves to even, or up by chance.
template <int BITS>
__device__ __forceinline__ uint32_t keep(float z, bool random, uint32_t h) {
  const uint32_t u = __float_as_uint(z);
  return (u + (random ? h : (1u << (BITS - 1)) - 1 + (u >> BITS & 1))) >> BITS;
}
struct Unit { float scale, inverse; bool number; };
// The power of two 2^BELOW under the largest power of two in `most` >= 0.
template <int BELOW>
__device__ __forceinline__ Unit unit_of(float most) {
  const int e = __float_as_int(most) >> 23, at = max(e - BELOW, 1);
  return e == 255 ? Unit{NAN, 0.f, false} : Unit{__int_as_float(at << 23), __int_as_float((254 - at) << 23), true};
}
// m: sign, four bits of exponent, three of mantissa (the 8-bit float e4m3), 256 at most.  Below 2^-6 a sum with it has the step of its smallest normal numbers.
__device__ __forceinline__ uint32_t code_m(float y, bool random, uint32_t h) {
  const float a = fabsf(y);
  const bool low = a < 0x1p-6f;
  return (keep<20>(low ? a + 0x1p-6f : a, random, h & 0xFFFFF) - (low ? 121 * 8 : 120 * 8)) | (__float_as_uint(y) >> 24 & 128);
}
__device__ __forceinline__ float value_m(uint32_t c) {
  const uint32_t a = c & 127;
  const float x = a < 8 ? a * 0x1p-9f : __uint_as_float((a + 120 * 8) << 20);
  return __uint_as_float((a == 127 ? 0x7FC00000u : __float_as_uint(x)) | (c & 128) << 24);
}
// sqrt v: four bits of exponent, four of mantissa, whole numbers below 32; what is above zero stays there, so that no m is divided by a lost v.
__device__ __forceinline__ uint32_t code_root(float y, bool some, bool random, uint32_t h) {
  const bool low = y < 16.f;
  const uint32_t c = keep<19>(low ? y + 16.f : y, random, (h * 0x9E3779B9u) >> 13) - (low ? 131 * 16 : 130 * 16);
  return some && c == 0 ? 1 : c;
}
__device__ __forceinline__ float value_root(uint32_t c) { return c < 16 ? (float)c : __uint_as_float((c + 130 * 16) << 19); }

__device__ __forceinline__ float largest_of_32(float x) {      // NaN where one is: the largest of the bits of what is not negative
  uint32_t u = __float_as_uint(x);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) { const uint32_t w = __shfl_xor(u, o, 32); u = w > u ? w : u; }
  return __uint_as_float(u);
}
typedef uint8_t u8x8 __attribute__((ext_vector_type(8)));
typedef u8x8 u8x8_any __attribute__((aligned(1)));
__device__ __forceinline__ u8x8 load_codes(const void* p, int64_t at, int64_t most) {
  const uint8_t* q = reinterpret_cast<const uint8_t*>(p) + at;
  if (most >= 8) return *reinterpret_cast<const u8x8_any*>(q);
  u8x8 w;
#pragma unroll
  for (int e = 0; e < 8; e++) { w[e] = 0; if (e < most) w[e] = q[e]; }
  return w;
}
__device__ __forceinline__ void store_codes(void* p, int64_t at, const u8x8& w, int64_t most) {
  uint8_t* q = reinterpret_cast<uint8_t*>(p) + at;
  if (most >= 8) { *reinterpret_cast<u8x8_any*>(q) = w; return; }
#pragma unroll
  for (int e = 0; e < 8; e++) if (e < most) q[e] = w[e];
}
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

// One pass over a chunk of one tensor, eight elements a thread.  Bound by reading and writing parameters and states.
template <bool P32, bool G32, bool MASTER, bool SMALL>
__global__ __launch_bounds__(T) void adamw_kernel(const Table<SMALL, MASTER> tab, const Step s, Factors f) {
  const int i = tensor_of(tab, blockIdx.x);
  const int64_t n = tab.n[i], at = (int64_t)(blockIdx.x - tab.begin[i]) * CHUNK + threadIdx.x * 8, most = n - at;
  const bool mine = most > 0;
  typedef Eight<P32 || MASTER> EP;
  typedef Eight<G32> EG;
  typename EP::type rp;
  typename EG::type rg;
  typename Eight<true>::type rm, rv;
  u8x8 cm, cv;
  float ms = 0.f, vs = 0.f;
  void* kept;
  if constexpr (MASTER) kept = tab.master[i];
  else kept = tab.p[i];
  if (mine) {
    rp = EP::load(kept, at, most);
    rg = EG::load(tab.g[i], at, most);
    if constexpr (SMALL) {
      cm = load_codes(tab.m[i], at, most);
      cv = load_codes(tab.v[i], at, most);
      ms = tab.m_scale[i][at / BLOCK];
      vs = tab.v_scale[i][at / BLOCK];
    } else {
      rm = Eight<true>::load(tab.m[i], at, most);
      rv = Eight<true>::load(tab.v[i], at, most);
    }
  }
  if (s.t_dev || s.lr_dev) f = factors_of(s, s.lr_dev ? (double)*s.lr_dev : s.lr, s.t_dev ? *s.t_dev : s.t);
  float gs = 1.f;
  if (s.scale_dev) {
    gs = *s.scale_dev;
    if (!(fabsf(gs) < INFINITY)) return;      // the step is left out
  }
  float p[8], g[8], m[8], v[8], root[8];
  if (mine) {
    EP::values(rp, p);
    EG::values(rg, g);
    if constexpr (!SMALL) {
      Eight<true>::values(rm, m);
      Eight<true>::values(rv, v);
    }
  }
#pragma unroll
  for (int e = 0; e < 8; e++) {
    if (!mine) { p[e] = g[e] = m[e] = v[e] = 0.f; }
    else if constexpr (SMALL) {
      m[e] = value_m(cm[e]) * ms;
      v[e] = value_root(cv[e]) * vs;
      v[e] = v[e] * v[e];
    }
    if (s.scale_dev) g[e] = g[e] * gs;
    m[e] = m[e] * f.b1 + g[e] * f.c1;
    v[e] = v[e] * f.b2 + (g[e] * g[e]) * f.c2;
    root[e] = sqrtf(v[e]);
    p[e] = p[e] * f.decay - f.step * (m[e] / (root[e] * f.root + s.eps));
  }
  uint32_t h[8];
  const bool random = s.random != 0;
  if (random) {
    const uint64_t number = (uint64_t)tab.first[i] * BLOCK + (uint64_t)at;      // of the element in the call; eight of them have one high half
    const uint32_t key = mix((uint32_t)(number >> 32) ^ mix(s.seed));
#pragma unroll
    for (int e = 0; e < 8; e++) h[e] = mix(((uint32_t)number + e) ^ key);
  } else {
#pragma unroll
    for (int e = 0; e < 8; e++) h[e] = 0;
  }
  if (mine) {
    EP::store(kept, at, p, most);
    if constexpr (!P32 && !MASTER) {
      if (random) {      // up by chance, as its part of a step is; again over what was rounded to the nearest
        uint16_t* q = reinterpret_cast<uint16_t*>(kept) + at;
        u16x8 w;
#pragma unroll
        for (int e = 0; e < 8; e++) w[e] = fabsf(p[e]) < INFINITY ? (uint16_t)((__float_as_uint(p[e]) + (h[e] >> 16)) >> 16) : bf16_nearest(p[e]);
        if (most >= 8) *reinterpret_cast<u16x8_any*>(q) = w;
        else {
#pragma unroll
          for (int e = 0; e < 8; e++) if (e < most) q[e] = w[e];
        }
      }
    }
    if constexpr (MASTER) Eight<false>::store(tab.p[i], at, p, most);
  }
  if constexpr (!SMALL) {
    if (mine) {
      Eight<true>::store(tab.m[i], at, m, most);
      Eight<true>::store(tab.v[i], at, v, most);
    }
  } else {
    float mm = 0.f, mr = 0.f;
#pragma unroll
    for (int e = 0; e < 8; e++) {      // (as bits, so that a NaN is the largest)
      mm = __uint_as_float(max(__float_as_uint(mm), e < most ? __float_as_uint(m[e]) & 0x7FFFFFFFu : 0u));
      mr = __uint_as_float(max(__float_as_uint(mr), e < most ? __float_as_uint(root[e]) & 0x7FFFFFFFu : 0u));
    }
    const Unit um = unit_of<7>(largest_of_32(mm)), ur = unit_of<17>(largest_of_32(mr));
    if (mine) {
#pragma unroll
      for (int e = 0; e < 8; e++) {
        cm[e] = um.number ? (uint8_t)code_m(m[e] * um.inverse, random, h[e]) : (uint8_t)0;
        cv[e] = ur.number ? (uint8_t)code_root(root[e] * ur.inverse, root[e] > 0.f, random, h[e]) : (uint8_t)0;
      }
      store_codes(tab.m[i], at, cm, most);
      store_codes(tab.v[i], at, cv, most);
      if ((threadIdx.x & 31) == 0) {
        tab.m_scale[i][at / BLOCK] = um.scale;
        tab.v_scale[i][at / BLOCK] = ur.scale;
      }
    }
  }
}

// What 8-bit states stand for, in bf16, which holds them exactly.
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
  const u8x8 cm = load_codes(tab.m[i], at, most), cv = load_codes(tab.v[i], at, most);
  const float ms = tab.m_scale[i][at / BLOCK], vs = tab.v_scale[i][at / BLOCK];
  float m[8], r[8];
#pragma unroll
  for (int e = 0; e < 8; e++) {
    m[e] = value_m(cm[e]) * ms;
    r[e] = value_root(cv[e]) * vs;
  }
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

template <bool P32, bool G32, bool MASTER, bool SMALL>
void steps(const osscar_adamw_tensor* t, int64_t count, const Step& s, const Factors& f, hipStream_t stream) {
  typedef Table<SMALL, MASTER> Tab;
  static_assert(sizeof(Tab) + sizeof(Step) + sizeof(Factors) <= 4096, "a launch's arguments");
  in_launches<Tab>(
      count, t, is_kind, (MASTER ? 2 : P32 ? 0 : 1) * 2 + (G32 ? 1 : 0),
      [](Tab& tab, int at, const osscar_adamw_tensor& x, int64_t number) {
        tab.p[at] = x.p;
        tab.g[at] = x.g;
        tab.m[at] = x.m;
        tab.v[at] = x.v;
        tab.n[at] = x.n;
        tab.first[at] = number;
        if constexpr (SMALL) { tab.m_scale[at] = x.m_scale; tab.v_scale[at] = x.v_scale; }
        if constexpr (MASTER) tab.master[at] = x.master;
      },
      [&](const Tab& tab, unsigned blocks) { hipLaunchKernelGGL((adamw_kernel<P32, G32, MASTER, SMALL>), dim3(blocks), dim3(T), 0, stream, tab, s, f); });
}
template <bool SMALL>
void steps_of(const osscar_adamw_tensor* t, int64_t count, const Step& s, const Factors& f, hipStream_t stream) {
  bool seen[6] = {};
  for (int64_t k = 0; k < count; k++)
    if (t[k].n > 0) seen[kind_of(t[k])] = true;
  if (seen[0]) steps<true, false, false, SMALL>(t, count, s, f, stream);
  if (seen[1]) steps<true, true, false, SMALL>(t, count, s, f, stream);
  if (seen[2]) steps<false, false, false, SMALL>(t, count, s, f, stream);
  if (seen[3]) steps<false, true, false, SMALL>(t, count, s, f, stream);
  if (seen[4]) steps<false, false, true, SMALL>(t, count, s, f, stream);
  if (seen[5]) steps<false, true, true, SMALL>(t, count, s, f, stream);
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
  const Step s{d->lr, d->beta1, d->beta2, d->weight_decay, (float)d->eps, 1.f, d->step, d->lr_dev, d->grad_scale_dev, d->step_dev, d->seed, d->stochastic != 0};
  const Factors f = factors_of(s, d->lr_dev ? 0 : d->lr, d->step_dev ? 1 : d->step);
  hipStream_t stream = reinterpret_cast<hipStream_t>(hip_stream);
  if (d->bits == 8) steps_of<true>(tensors, count, s, f, stream);
  else steps_of<false>(tensors, count, s, f, stream);
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
