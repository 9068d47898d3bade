// Gated feed-forward: g = X Wg, u = X Wu, h = a(g) u with a one of SiLU, GELU (two forms), ReLU; its backward pass
//     dg = dh u a'(g), du = dh a(g);   dX = dg Wg^T + du Wu^T, dWg = X^T dg, dWu = X^T du.
// h is the X that the Gram of the layer's down projection takes.  Both projections are one product with the activation in its epilogue, both gradients of the
// weights one launch, dX one sum over both.  bf16, 16384 x 2048 x 8192 forward 0.88 to 0.94 ms by machine (1170 to 1250 TFLOP/s), 4096 x 7168 x 14336 forward
// with g and u kept and backward 4.0 to 4.3 ms (1170 to 1260).
#include "ops.h"
#include "split.h"
#include "thin.h"
#include "tile.h"
#include <algorithm>

using namespace osscar;
using namespace osscar::tile;

namespace {

// ---- activations -----------------------------------------------------------------------------
// logistic function; e^-x past float32's range gives 0
__device__ __forceinline__ float logistic(float x) { return __builtin_amdgcn_rcpf(1.f + __expf(-x)); }
constexpr float ROOT_HALF = 0.70710678118654752f, TWO_ROOT_2_PI = 1.5957691216057308f, ROOT_2PI_INV = 0.39894228040143268f;
// The normal distribution function at g, and e = exp(-g^2 / 2).  With x = |g| / sqrt 2 and t = 1 / (1 + 0.45 x), erfc(x) = t P(t) exp(-x^2): erfc(x) exp(x^2) / t is
// smooth in t on (0, 1], P its Chebyshev fit of degree nine (relative error 3e-8; with float32's own rounding 7e-7 where erfc is not negligible, both
// signs).  The math library's erf cost an epilogue of 128 values a lane 17 us.
__device__ __forceinline__ float normal_cdf(float g, float& e) {
  const float x = fabsf(g) * ROOT_HALF, t = __builtin_amdgcn_rcpf(1.f + 0.45f * x), s = 2.f * t - 1.f;
  float p = -8.13252922e-05f;
  p = fmaf(p, s, 1.68057889e-05f); p = fmaf(p, s, 0.000701177373f); p = fmaf(p, s, -0.000146496056f);
  p = fmaf(p, s, -0.00513639725f); p = fmaf(p, s, -0.00285712009f); p = fmaf(p, s, 0.0421393369f);
  p = fmaf(p, s, 0.162789169f); p = fmaf(p, s, 0.335434536f); p = fmaf(p, s, 0.467140291f);
  e = __expf(-x * x);
  const float h = 0.5f * t * p * e;
  return g > 0.f ? 1.f - h : h;
}

template <int ACT>
__device__ __forceinline__ float act_value(float g) {
  if (ACT == OSSCAR_ACT_SILU) return g * logistic(g);
  if (ACT == OSSCAR_ACT_GELU) { float e; return g * normal_cdf(g, e); }
  if (ACT == OSSCAR_ACT_GELU_TANH) return g * logistic(TWO_ROOT_2_PI * (g + 0.044715f * g * g * g));      // (1 + tanh(w / 2)) / 2 is the logistic function of w
  return g > 0.f ? g : (g == g ? 0.f : g);      // NaN stays
}
template <int ACT>
__device__ __forceinline__ void act_slope(float g, float& a, float& da) {
  if (ACT == OSSCAR_ACT_SILU) {
    const float s = logistic(g);
    a = g * s;
    da = s + a * (1.f - s);
  } else if (ACT == OSSCAR_ACT_GELU) {
    float e;
    const float c = normal_cdf(g, e);
    a = g * c;
    da = c + g * e * ROOT_2PI_INV;
  } else if (ACT == OSSCAR_ACT_GELU_TANH) {
    const float s = logistic(TWO_ROOT_2_PI * (g + 0.044715f * g * g * g));
    a = g * s;
    da = s + a * (1.f - s) * TWO_ROOT_2_PI * (1.f + 3.f * 0.044715f * fminf(g * g, 1e30f));      // (no infinity to multiply the 0 with)
  } else {
    a = act_value<OSSCAR_ACT_RELU>(g);
    da = g > 0.f ? 1.f : (g == g ? 0.f : g);
  }
}
// f(integral_constant) for the activation of a call
template <class F>
__device__ __forceinline__ void with_act(int act, F f) {
  switch (act) {
    case OSSCAR_ACT_SILU: f(std::integral_constant<int, OSSCAR_ACT_SILU>()); break;
    case OSSCAR_ACT_GELU: f(std::integral_constant<int, OSSCAR_ACT_GELU>()); break;
    case OSSCAR_ACT_GELU_TANH: f(std::integral_constant<int, OSSCAR_ACT_GELU_TANH>()); break;
    default: f(std::integral_constant<int, OSSCAR_ACT_RELU>());
  }
}

// ---- copies ----------------------------------------------------------------------------------
// Up to three bf16 matrices (blockIdx.y) with rows of `ld` (a multiple of eight), zeros past cols.  Eight columns per thread; bound by its reads and writes.
struct Copies { struct { const uint16_t* src; int64_t rows, lds; int cols; uint16_t* dst; int64_t ld; } m[3]; };
__global__ __launch_bounds__(256) void gated_copy_kernel(const Copies q) {
  const auto& m = q.m[blockIdx.y];
  const int packs = (int)(m.ld / 8);
  for (int64_t i = blockIdx.x * (int64_t)256 + threadIdx.x; i < m.rows * packs; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / packs;
    const int c = (int)(i - r * packs) * 8;
    u16x8 w;
    if (c + 8 <= m.cols) {
      w = *reinterpret_cast<const u16x8_any*>(m.src + r * m.lds + c);
    } else {
#pragma unroll
      for (int e = 0; e < 8; e++) {
        w[e] = 0;
        if (c + e < m.cols) w[e] = m.src[r * m.lds + c + e];
      }
    }
    *reinterpret_cast<u16x8*>(m.dst + r * m.ld + c) = w;
  }
}

// ---- epilogues -------------------------------------------------------------------------------
struct GatedOut {      // h, and g and u as they are where the caller keeps them for the backward pass; H may be NULL then
  void* H; int64_t ldh; int f32, act; float *G, *U;
  template <class F>
  __device__ __forceinline__ void each(F f) const {
    with_act(H ? act : OSSCAR_ACT_RELU, [&](auto a) {
      f([&](int m, int n, const float (&v)[2][8], int N) {
        if (H) {
          float h[8];
#pragma unroll
          for (int c = 0; c < 8; c++) h[c] = act_value<decltype(a)::value>(v[0][c]) * v[1][c];
          if (f32) put_f32(reinterpret_cast<float*>(H) + (int64_t)m * ldh + n, h, N - n);
          else put_bf16(reinterpret_cast<uint16_t*>(H) + (int64_t)m * ldh + n, h, N - n);
        }
        if (G) {
          put_f32(G + (int64_t)m * N + n, v[0], N - n);
          put_f32(U + (int64_t)m * N + n, v[1], N - n);
        }
      });
    });
  }
  template <class F>
  __device__ __forceinline__ void one(F f) const {
    with_act(H ? act : OSSCAR_ACT_RELU, [&](auto a) {
      f([&](int m, int n, const float (&v)[2], int N) {
        if (H) {
          const float h = act_value<decltype(a)::value>(v[0]) * v[1];
          if (f32) reinterpret_cast<float*>(H)[(int64_t)m * ldh + n] = h;
          else reinterpret_cast<uint16_t*>(H)[(int64_t)m * ldh + n] = bf16_nearest(h);
        }
        if (G) { G[(int64_t)m * N + n] = v[0]; U[(int64_t)m * N + n] = v[1]; }
      });
    });
  }
};
template <int LAYOUT, int KIND, int RT, bool WIDE>
__global__ __launch_bounds__((thin::Wave<LAYOUT, KIND, 2, RT, WIDE>::WAVES) * 64, 1) void gated_thin_kernel(const thin::Product<2> p, const GatedOut e) {
  thin::product<LAYOUT, KIND, 2, RT, WIDE>(p, e);
}
__global__ __launch_bounds__(256) void gated_join_kernel(const float* __restrict__ sums, int parts, int M, int N, const GatedOut e) {
  tile::join<2>(sums, parts, M, N, e);
}

struct PlainOut {
  void* out; int64_t ld; int f32;
  template <class F>
  __device__ __forceinline__ void each(F f) const {
    f([&](int m, int n, const float (&v)[1][8], int N) {
      if (f32) put_f32(reinterpret_cast<float*>(out) + (int64_t)m * ld + n, v[0], N - n);
      else put_bf16(reinterpret_cast<uint16_t*>(out) + (int64_t)m * ld + n, v[0], N - n);
    });
  }
};
// dg and du from kept g and u, in the type of the products that take them: bf16 rounds them once more, as h is rounded for the next layer.  Rows of
// `ld`, a multiple of eight, zeros past f.  Bound by its 14 (float32: 20) bytes per element: 4096 x 14336 bf16 154 us, 5.3 TB/s.
template <bool F32>
__global__ __launch_bounds__(256) void gated_grad_kernel(const void* __restrict__ dH, int64_t lddh, int act, const float* __restrict__ G,
                                                         const float* __restrict__ U, int64_t rows, int f, void* __restrict__ out_g, void* __restrict__ out_u, int64_t ld) {
  const int packs = (int)(ld / 8);
  for (int64_t i = blockIdx.x * (int64_t)256 + threadIdx.x; i < rows * packs; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / packs;
    const int n = (int)(i - r * packs) * 8;
    float g[8], u[8], dh[8];
    get_values(G, r * f + n, 1, g, f - n);
    get_values(U, r * f + n, 1, u, f - n);
    get_values(dH, r * lddh + n, F32, dh, f - n);
    float dg[8], du[8];
    with_act(act, [&](auto a) {
#pragma unroll
      for (int c = 0; c < 8; c++) {
        float av, da;
        act_slope<decltype(a)::value>(g[c], av, da);
        const bool in = n + c < f;
        dg[c] = in ? dh[c] * u[c] * da : 0.f;
        du[c] = in ? dh[c] * av : 0.f;
      }
    });
    const int64_t at = r * ld + n;
    if (F32) {
      put_f32(reinterpret_cast<float*>(out_g) + at, dg, 8);
      put_f32(reinterpret_cast<float*>(out_u) + at, du, 8);
    } else {
      put_bf16(reinterpret_cast<uint16_t*>(out_g) + at, dg, 8);
      put_bf16(reinterpret_cast<uint16_t*>(out_u) + at, du, 8);
    }
  }
}

// up to two products of the same sizes in one launch
template <int NB, class Epi> struct Pair { Product<NB> p[2]; Epi e[2]; };
template <int AM, int BMODE, class S, class Epi>
__global__ __launch_bounds__(S::WAVES * 64, 1) void gated_product_kernel(const Pair<S::NB, Epi> q) {
  tile::product_tile<false, AM, BMODE, S>(q.p[blockIdx.y], q.e[blockIdx.y]);
}
template <int AM, int BMODE, class S, class Epi>      // float32
__global__ __launch_bounds__(S::WAVES * 64, 2) void gated_split_kernel(const Pair<S::NB, Epi> q) {
  split::product_tile<AM, BMODE, S>(q.p[blockIdx.y], q.e[blockIdx.y]);
}

// ---- shapes ----------------------------------------------------------------------------------
typedef Shape<2, 2, 8, 4, 2> Big2;       // 256 x (128 + 128), four waves
typedef Shape<2, 2, 4, 2, 2> Small2;     // 128 x (64 + 64), four waves
typedef Shape<2, 2, 8, 8, 1> Big1;       // 256 x 256
typedef Shape<2, 2, 4, 4, 1> Small1;     // 128 x 128
typedef Shape<1, 4, 4, 2, 2> Flat2;      // 64 x (128 + 128)
typedef Shape<1, 4, 4, 4, 1> Flat1;      // 64 x 256
template <class S, int G, class Epi>
__global__ __launch_bounds__(256) void gated_join_tiles_kernel(const Pair<S::NB, Epi> q) {
  tile::join_tiles<S, float, G>(q.p[blockIdx.y], q.e[blockIdx.y]);
}
template <class S, class Epi>
void launch_join(const Pair<S::NB, Epi>& q, int count, const Deal& d, hipStream_t s) {
  const dim3 grid((unsigned)d.join, count);
  if (d.parts >= JOIN_GROUPS_FROM) hipLaunchKernelGGL((gated_join_tiles_kernel<S, 4, Epi>), grid, dim3(256), 0, s, q);
  else hipLaunchKernelGGL((gated_join_tiles_kernel<S, 1, Epi>), grid, dim3(256), 0, s, q);
}
// `count` products of one launch; sums: d.sums for each
template <int AM, int BMODE, class SB, class SS, class SF, class Epi>
void launch_product(Pair<SB::NB, Epi>& q, int count, bool f32, const Deal& d, char* sums, hipStream_t s) {
  for (int c = 0; c < count; c++) {
    q.p[c].whole = d.whole;
    q.p[c].parts = d.parts;
    q.p[c].sums = sums + c * d.sums;
  }
  const dim3 grid(d.blocks, count);
  if constexpr (AM == OP_K)
    if (d.pick == FLAT) hipLaunchKernelGGL((gated_split_kernel<AM, BMODE, SF, Epi>), grid, dim3(SF::WAVES * 64), 0, s, q);
  if (d.pick == SMALL && f32) hipLaunchKernelGGL((gated_split_kernel<AM, BMODE, SS, Epi>), grid, dim3(SS::WAVES * 64), 0, s, q);
  else if (d.pick == BIG_TILE) hipLaunchKernelGGL((gated_product_kernel<AM, BMODE, SB, Epi>), grid, dim3(SB::WAVES * 64), 0, s, q);
  else if (d.pick == SMALL) hipLaunchKernelGGL((gated_product_kernel<AM, BMODE, SS, Epi>), grid, dim3(SS::WAVES * 64), 0, s, q);
  if (d.parts < 2) return;
  if (d.pick == FLAT) launch_join<SF>(q, count, d, s);
  else if (d.pick == BIG_TILE) launch_join<SB>(q, count, d, s);
  else launch_join<SS>(q, count, d, s);
}

// ---- operands --------------------------------------------------------------------------------
inline int64_t up8(int64_t v) { return (v + 7) / 8 * 8; }
inline unsigned packs_grid(int64_t rows, int64_t ld) {
  const int64_t n = (rows * (ld / 8) + 255) / 256;
  return (unsigned)(n < 1 ? 1 : (n > 8192 ? 8192 : n));
}
// A matrix of a call as the products take it: in place, or (bf16 at other alignments) copied to the workspace.
struct Source {
  const void* p; int64_t rows, cols, ld; int es; bool copied; char* at;
  Operand operand() const {
    Operand o{};
    o.p[0] = copied ? at : reinterpret_cast<const char*>(p);
    o.ldb = (copied ? up8(cols) : ld) * es; o.rows = (int)rows; o.cols = (int)(copied ? up8(cols) : cols);
    return o;
  }
};
// Makes the copies that these need, in one launch.
void make_copies(const Source* const (&from)[3], hipStream_t s) {
  Copies q{};
  int n = 0;
  unsigned grid = 1;
  for (const Source* f : from)
    if (f && f->copied && f->rows > 0) {
      const int64_t ld = up8(f->cols);
      q.m[n].src = reinterpret_cast<const uint16_t*>(f->p); q.m[n].rows = f->rows; q.m[n].lds = f->ld; q.m[n].cols = (int)f->cols;
      q.m[n].dst = reinterpret_cast<uint16_t*>(f->at); q.m[n].ld = ld;
      const unsigned need = packs_grid(f->rows, ld);
      grid = grid > need ? grid : need;
      n++;
    }
  if (n > 0) hipLaunchKernelGGL(gated_copy_kernel, dim3(grid, n), dim3(256), 0, s, q);
}
// `loose`: some buffer of the call does not begin at a 16-byte boundary
Source source(Carve& c, const void* p, int64_t rows, int64_t cols, int64_t ld, int32_t dtype, bool loose) {
  Source s{p, rows, cols, ld, dtype == OSSCAR_F32 ? 4 : 2, false, nullptr};
  s.copied = dtype == OSSCAR_BF16 && (loose || !operand_fits(nullptr, ld, cols, 2));
  if (s.copied) s.at = c.take((size_t)rows * up8(cols) * 2);
  return s;
}
template <int NB>
void add_segment(Product<NB>& q, const Operand& a, const Operand (&b)[NB]) {
  q.a.ldb = a.ldb; q.a.rows = a.rows; q.a.cols = a.cols;
  q.a.p[q.nseg] = a.p[0];
  for (int z = 0; z < NB; z++) {
    q.b[z].ldb = b[z].ldb; q.b[z].rows = b[z].rows; q.b[z].cols = b[z].cols;
    q.b[z].p[q.nseg] = b[z].p[0];
  }
  q.nseg++;
}

struct Buffers {
  Source x, wg, wu;
  char *dg, *du; int64_t ldg;
  float *g, *u;      // computed again
  thin::Deal few;        // how the products are dealt out: few rows' projections, others', dX, both weights' gradients
  Deal proj, dx, dw;
  char* sums;            // of parts, one product after the other
  bool launchable() const {
    return osscar::launchable(few.blocks, few.threads) && osscar::launchable(proj.blocks, 256) && osscar::launchable(dx.blocks, 256) && osscar::launchable(dw.blocks, 256);
  }
};
const char TOO_LARGE[] = "osscar_gated: the products of the sizes are too large for one call";
// The products of few rows (thin.h says where)
bool few(const osscar_gated_desc& q) {
  if (q.dtype == OSSCAR_F32) return q.n <= 16 || (q.n <= 32 && q.d * q.f <= (1 << 25));
  return q.rows_out && q.n <= 16 && (q.d * q.f <= (1 << 24) || q.unaligned || !operand_fits(nullptr, q.ldw, q.d, 2));
}
Buffers buffers(Carve& c, const osscar_gated_desc& q, const void* X, const void* Wg, const void* Wu, int backward, bool kept) {
  Buffers b{};
  const bool f32 = q.dtype == OSSCAR_F32;
  const int ks = f32 ? split::KS : STEP_BYTES / 2;
  size_t sums = 0;
  if (!kept && few(q)) {
    b.few = !f32 ? thin::deal<OP_K, thin::BF16>(q.n, q.f, q.d) : q.rows_out ? thin::deal<OP_K, thin::F32>(q.n, q.f, q.d) : thin::deal<OP_T, thin::F32>(q.n, q.f, q.d);
    if (b.few.parts > 1) sums = (size_t)b.few.parts * 2 * q.n * q.f * 4;
    if (q.n == 0) b.few.blocks = 0;
  } else if (!kept) {
    const int64_t stages = (q.d + ks - 1) / ks;
    b.proj = f32 ? deal_split<Flat2, Small2>(q.n, q.f, stages, 1, true) : deal<Big2, Small2>(q.n, q.f, stages, 1);
    sums = b.proj.sums;
  }
  if (backward) {
    const int64_t sx = (q.f + ks - 1) / ks * 2, sw = (q.n + ks - 1) / ks, M = q.rows_out ? q.f : q.d, N = q.rows_out ? q.d : q.f;
    b.dx = f32 ? deal_split<Flat1, Small1>(q.n, q.d, sx, 1, true) : deal<Big1, Small1>(q.n, q.d, sx, 1);
    b.dw = f32 ? deal_split<Flat1, Small1>(M, N, sw, 2, false) : deal<Big1, Small1>(M, N, sw, 2);
    sums = sums > b.dx.sums ? sums : b.dx.sums;
    sums = sums > 2 * b.dw.sums ? sums : 2 * b.dw.sums;
  }
  b.sums = c.take(sums);
  if (!backward && few(q)) return b;
  const int64_t wr = q.rows_out ? q.f : q.d, wc = q.rows_out ? q.d : q.f;
  b.x = source(c, X, q.n, q.d, q.ldx, q.dtype, q.unaligned != 0);
  b.wg = source(c, Wg, wr, wc, q.ldw, q.dtype, q.unaligned != 0);
  b.wu = source(c, Wu, wr, wc, q.ldw, q.dtype, q.unaligned != 0);
  if (backward) {
    b.ldg = up8(q.f);
    const size_t bytes = (size_t)q.n * b.ldg * (q.dtype == OSSCAR_F32 ? 4 : 2);
    b.dg = c.take(bytes);
    b.du = c.take(bytes);
    if (!kept) {
      b.g = reinterpret_cast<float*>(c.take((size_t)q.n * q.f * 4));
      b.u = reinterpret_cast<float*>(c.take((size_t)q.n * q.f * 4));
    }
  }
  return b;
}
// Whether the tiles reach all of every bf16 operand: rows as long as the copies and dg, du have them, along the contraction and across it
bool addressable(const osscar_gated_desc& q, int backward, bool kept) {
  if (q.dtype == OSSCAR_F32 || q.n == 0) return true;
  const int64_t along = std::max(kept || few(q) ? 0 : q.d, backward ? q.f : 0);
  const int64_t across = std::max(!q.rows_out && !kept && !few(q) ? q.f : 0, backward ? std::max(q.d, q.f) : 0);
  return up8(along) * 2 <= MAX_K_BYTES && up8(across) * 2 <= MAX_T_BYTES;
}
const char TOO_LONG[] = "osscar_gated: rows of the bf16 operands are too long (d, and f of a backward pass: 4194296; f of a forward pass: 16777208)";
int64_t up_tiles(int64_t v) { return (v + 63) / 64; }
const char* bad_desc(const osscar_gated_desc* q) {
  if (!q) return "osscar_gated: NULL description";
  if (!a_size(q->n, 0) || !a_size(q->d, 1) || !a_size(q->f, 1)) return "osscar_gated: n >= 0, d and f must be positive, none above 2^30";
  if (up_tiles(q->n) * up_tiles(q->f) > 0x3FFFFFFF || up_tiles(q->n) * up_tiles(q->d) > 0x3FFFFFFF || up_tiles(q->d) * up_tiles(q->f) > 0x3FFFFFFF)
    return TOO_LARGE;
  if (!real_dtype(q->dtype)) return "osscar_gated: unknown dtype";
  if (q->act < OSSCAR_ACT_SILU || q->act > OSSCAR_ACT_RELU) return "osscar_gated: unknown activation";
  if (q->ldx < q->d || q->ldw < (q->rows_out ? q->d : q->f) || q->ldh < q->f) return "osscar_gated: leading dimension below the row length";
  return nullptr;
}
bool loose(const void* p) { return ((uintptr_t)p & 15) != 0; }
// what both calls check of their buffers; nullptr if there is nothing to refuse
const char* bad_buffers(const osscar_gated_desc& q, const void* X, const void* Wg, const void* Wu, const void* H, const void* G, const void* U, const void* ws) {
  if (!Wg || !Wu || (q.n > 0 && (!X || !H))) return "osscar_gated: NULL pointer";
  if ((G == nullptr) != (U == nullptr) && q.n > 0) return "osscar_gated: G and U are given together or not at all";
  const uintptr_t es = q.dtype == OSSCAR_F32 ? 4 : 2;
  if ((uintptr_t)X % es || (uintptr_t)Wg % es || (uintptr_t)Wu % es || (uintptr_t)H % es || (uintptr_t)G % 4 || (uintptr_t)U % 4)
    return "osscar_gated: a buffer is not aligned to its elements";
  if (q.dtype == OSSCAR_BF16 && !q.unaligned && (loose(X) || loose(Wg) || loose(Wu)))
    return "osscar_gated: X, Wg or Wu does not begin at a 16-byte boundary (set unaligned in the description)";
  if ((uintptr_t)ws & 255) return "osscar_gated: the workspace must begin at a 256-byte boundary";
  return nullptr;
}

template <int LAYOUT, int KIND, int RT, bool WIDE>
void thin_launch(const thin::Product<2>& p, const thin::Deal& d, const GatedOut& e, hipStream_t s) {
  hipLaunchKernelGGL((gated_thin_kernel<LAYOUT, KIND, RT, WIDE>), dim3(d.blocks, (unsigned)d.parts), dim3(thin::Wave<LAYOUT, KIND, 2, RT, WIDE>::WAVES * 64), 0, s, p, e);
}
void thin_projections(const thin::Product<2>& p, bool f32, bool rows_out, const thin::Deal& d, const GatedOut& e, hipStream_t s) {
  const bool one = p.M <= 16;
  if (!f32) thin_launch<OP_K, thin::BF16, 1, false>(p, d, e, s);
  else if (!rows_out) one ? thin_launch<OP_T, thin::F32, 1, false>(p, d, e, s) : thin_launch<OP_T, thin::F32, 2, false>(p, d, e, s);
  else if (d.wide) one ? thin_launch<OP_K, thin::F32, 1, true>(p, d, e, s) : thin_launch<OP_K, thin::F32, 2, true>(p, d, e, s);
  else one ? thin_launch<OP_K, thin::F32, 1, false>(p, d, e, s) : thin_launch<OP_K, thin::F32, 2, false>(p, d, e, s);
  if (d.parts > 1)
    hipLaunchKernelGGL(gated_join_kernel, dim3(join_grid(p.M, p.N)), dim3(256), 0, s, reinterpret_cast<const float*>(p.sums), d.parts, p.M, p.N, e);
}
// X Wg, X Wu with epilogue e
void projections(const osscar_gated_desc& q, const Buffers& b, const void* X, const void* Wg, const void* Wu, const GatedOut& e, hipStream_t s) {
  if (few(q)) {
    const int es = q.dtype == OSSCAR_F32 ? 4 : 2;
    const thin::Product<2> p{reinterpret_cast<const char*>(X), {reinterpret_cast<const char*>(Wg), reinterpret_cast<const char*>(Wu)}, q.ldx * es, q.ldw * es,
                             (int)q.n, (int)q.f, (int)q.d, b.few.parts, b.sums};
    thin_projections(p, q.dtype == OSSCAR_F32, q.rows_out != 0, b.few, e, s);
    return;
  }
  Pair<2, GatedOut> two{};
  Product<2>& p = two.p[0];
  two.e[0] = e;
  p.M = (int)q.n; p.N = (int)q.f; p.k = (int)q.d;
  const Operand w[2] = {b.wg.operand(), b.wu.operand()};
  add_segment(p, b.x.operand(), w);
  if (q.rows_out) launch_product<OP_K, OP_K, Big2, Small2, Flat2>(two, 1, e.f32, b.proj, b.sums, s);
  else launch_product<OP_K, OP_T, Big2, Small2, Flat2>(two, 1, e.f32, b.proj, b.sums, s);
}

}  // namespace

extern "C" size_t osscar_gated_workspace_bytes(const osscar_gated_desc* desc, int32_t backward) {
  if (bad_desc(desc) || !addressable(*desc, backward != 0, backward == 1)) return 0;
  Carve c(nullptr);
  if (!buffers(c, *desc, nullptr, nullptr, nullptr, backward != 0, backward == 1).launchable()) return 0;
  return c.used + 256;      // (never 0: that says that the description is invalid)
}

extern "C" osscar_status osscar_gated_forward(const osscar_gated_desc* desc, const void* X_dev, const void* Wg_dev, const void* Wu_dev, void* H_dev,
                                              float* G_dev, float* U_dev, void* workspace_dev, size_t workspace_bytes, void* hip_stream) {
  const char* bad = bad_desc(desc);
  if (!bad) bad = bad_buffers(*desc, X_dev, Wg_dev, Wu_dev, H_dev, G_dev, U_dev, workspace_dev);
  if (!bad && !addressable(*desc, 0, false)) bad = TOO_LONG;
  if (bad) return refuse_call(OSSCAR_EINVAL, bad);
  const osscar_gated_desc& q = *desc;
  Carve c(workspace_dev);
  const Buffers b = buffers(c, q, X_dev, Wg_dev, Wu_dev, 0, false);
  if (!b.launchable()) return refuse_call(OSSCAR_EINVAL, TOO_LARGE);
  if (c.used > workspace_bytes || (c.used > 0 && !workspace_dev)) return refuse_call(OSSCAR_ENOMEM, "osscar_gated_forward: workspace too small");
  if (q.n == 0) return OSSCAR_OK;
  hipStream_t s = reinterpret_cast<hipStream_t>(hip_stream);
  const int f32 = q.dtype == OSSCAR_F32;
  if (!few(q)) make_copies({&b.x, &b.wg, &b.wu}, s);
  const GatedOut e{H_dev, q.ldh, f32, q.act, G_dev, U_dev};
  projections(q, b, X_dev, Wg_dev, Wu_dev, e, s);
  return launched();
}

extern "C" osscar_status osscar_gated_backward(const osscar_gated_desc* desc, const void* X_dev, const void* Wg_dev, const void* Wu_dev, const void* dH_dev,
                                               const float* G_dev, const float* U_dev, void* dX_dev, int64_t lddx, void* dWg_dev, void* dWu_dev, int64_t lddw,
                                               int32_t dw_dtype, void* workspace_dev, size_t workspace_bytes, void* hip_stream) {
  const char* bad = bad_desc(desc);
  if (!bad) bad = bad_buffers(*desc, X_dev, Wg_dev, Wu_dev, dH_dev, G_dev, U_dev, workspace_dev);
  if (!bad && !addressable(*desc, 1, G_dev != nullptr)) bad = TOO_LONG;
  if (!bad && (!real_dtype(dw_dtype) || (dWg_dev == nullptr) != (dWu_dev == nullptr))) bad = "osscar_gated_backward: unknown dtype, or one of dWg and dWu alone";
  if (!bad && ((dX_dev && lddx < desc->d) || (dWg_dev && lddw < (desc->rows_out ? desc->d : desc->f))))
    bad = "osscar_gated_backward: leading dimension below the row length";
  if (!bad && ((uintptr_t)dX_dev % (desc->dtype == OSSCAR_F32 ? 4 : 2) || (uintptr_t)dWg_dev % (dw_dtype == OSSCAR_F32 ? 4 : 2) || (uintptr_t)dWu_dev % (dw_dtype == OSSCAR_F32 ? 4 : 2)))
    bad = "osscar_gated_backward: a buffer is not aligned to its elements";
  if (bad) return refuse_call(OSSCAR_EINVAL, bad);
  const osscar_gated_desc& q = *desc;
  Carve c(workspace_dev);
  const Buffers b = buffers(c, q, X_dev, Wg_dev, Wu_dev, 1, G_dev != nullptr);
  if (!b.launchable()) return refuse_call(OSSCAR_EINVAL, TOO_LARGE);
  if (c.used > workspace_bytes || (c.used > 0 && !workspace_dev)) return refuse_call(OSSCAR_ENOMEM, "osscar_gated_backward: workspace too small");
  hipStream_t s = reinterpret_cast<hipStream_t>(hip_stream);
  const int f32 = q.dtype == OSSCAR_F32;
  if (q.n > 0) {
    const bool x = !G_dev || dWg_dev, w = !G_dev || dX_dev;
    make_copies({x ? &b.x : nullptr, w ? &b.wg : nullptr, w ? &b.wu : nullptr}, s);
    const float *G = G_dev, *U = U_dev;
    if (!G) {
      projections(q, b, X_dev, Wg_dev, Wu_dev, GatedOut{nullptr, 0, f32, q.act, b.g, b.u}, s);
      G = b.g; U = b.u;
    }
    const dim3 grid(packs_grid(q.n, b.ldg));
    if (f32) hipLaunchKernelGGL(gated_grad_kernel<true>, grid, dim3(256), 0, s, dH_dev, q.ldh, q.act, G, U, q.n, (int)q.f, b.dg, b.du, b.ldg);
    else hipLaunchKernelGGL(gated_grad_kernel<false>, grid, dim3(256), 0, s, dH_dev, q.ldh, q.act, G, U, q.n, (int)q.f, b.dg, b.du, b.ldg);
  }
  // dg and du as operands: n rows of ldg, zeros past f
  Operand dg{}, du{};
  dg.p[0] = b.dg; du.p[0] = b.du;
  dg.ldb = du.ldb = b.ldg * (f32 ? 4 : 2); dg.rows = du.rows = (int)q.n; dg.cols = du.cols = (int)b.ldg;
  if (dX_dev && q.n > 0) {
    Pair<1, PlainOut> two{};
    Product<1>& p = two.p[0];
    p.M = (int)q.n; p.N = (int)q.d; p.k = (int)q.f;
    const Operand wg[1] = {b.wg.operand()}, wu[1] = {b.wu.operand()};
    add_segment(p, dg, wg);
    add_segment(p, du, wu);
    two.e[0] = PlainOut{dX_dev, lddx, f32};
    if (q.rows_out) launch_product<OP_K, OP_T, Big1, Small1, Flat1>(two, 1, f32, b.dx, b.sums, s);
    else launch_product<OP_K, OP_K, Big1, Small1, Flat1>(two, 1, f32, b.dx, b.sums, s);
  }
  if (dWg_dev) {      // both weights in one launch
    Pair<1, PlainOut> two{};
    Product<1>* p = two.p;
    const Operand x = b.x.operand(), *dd[2] = {&dg, &du};
    for (int z = 0; z < 2; z++) {
      const Operand bs[1] = {q.rows_out ? x : *dd[z]};
      add_segment(p[z], q.rows_out ? *dd[z] : x, bs);
      p[z].M = (int)(q.rows_out ? q.f : q.d); p[z].N = (int)(q.rows_out ? q.d : q.f); p[z].k = (int)q.n;
    }
    two.e[0] = PlainOut{dWg_dev, lddw, dw_dtype == OSSCAR_F32};
    two.e[1] = PlainOut{dWu_dev, lddw, dw_dtype == OSSCAR_F32};
    launch_product<OP_T, OP_T, Big1, Small1, Flat1>(two, 2, f32, b.dw, b.sums, s);
  }
  return launched();
}
