// Layer norm of rows and its gradients.
#include "ops.h"
#include <float.h>

// Products and sums are rounded each, but where fmaf says otherwise: the mean that is kept has to be the one that was taken off (a row of one value is then zero in the backward pass too).
#pragma clang fp contract(off)

using namespace osscar;

namespace {

// A row is read once and stays in registers: TPR threads hold PK packets of eight columns each, thread t those at (k TPR + t) 8; the last packet of a row that is no
// multiple of eight long begins eight before its end, and the columns that it shares with the one before are counted there (and written twice, the same).
// The mean first, then the squares of what is left of it (two passes over registers, so that a large mean costs no digits); the rounding of the mean, which every
// difference has, is summed beside them and taken out.  Sums are float32.
// Rows shorter than a packet or longer than the longest shape are read three times (the second and third time from the cache, as far as it holds them).
constexpr int LONGEST = 1024 * 8 * 2;
// Where packet k of thread t lies, and how many of its columns the packet before has
template <int TPR>
struct Place {
  int at, skip;
  bool in;
  __device__ __forceinline__ Place(int k, int tid, int d) {
    const int begin = (k * TPR + tid) * 8;
    at = min(begin, d - 8);
    skip = begin - at;
    in = begin < d;
  }
};

template <int TPR, int GROUPS>
__device__ __forceinline__ void sum2(float& a, float& b, float2* sh, int sub, int tid) {      // over the TPR threads of a row; sh: GROUPS x TPR / 64
#pragma unroll
  for (int o = (TPR < 64 ? TPR : 64) / 2; o > 0; o >>= 1) { a += __shfl_xor(a, o, 64); b += __shfl_xor(b, o, 64); }
  if constexpr (TPR > 64) {
    constexpr int W = TPR / 64;
    __syncthreads();
    if ((tid & 63) == 0) sh[sub * W + (tid >> 6)] = float2{a, b};
    __syncthreads();
    a = b = 0.f;
#pragma unroll
    for (int w = 0; w < W; w++) { a += sh[sub * W + w].x; b += sh[sub * W + w].y; }
  }
}
// A sum of squares past float32 has no norm here: NaN rather than zeros
__device__ __forceinline__ float rstd_of(float var, float eps) { return var < INFINITY ? 1.f / sqrtf(fmaxf(var, 0.f) + eps) : NAN; }

struct Rows { int64_t n; int d; int64_t ldx, ldy; };
struct Affine { const void *w, *b; int f32; float eps; };      // (w, b may be NULL)

__device__ __forceinline__ void affine_values(const void* p, int f32, int at, int d, float (&v)[8], float missing) {
  if (p) get_values(p, at, f32, v, d - at);
  else {
#pragma unroll
    for (int e = 0; e < 8; e++) v[e] = missing;
  }
}

// Forward.  Bound by reading X and writing Y: bf16 16384 x 2048 25 us (5.4 TB/s), 8192 x 7168 45 us (5.2), 100000 x 64 7 us (3.5), 4096 x 14336 60 us (3.9; one workgroup of 1024
// threads a compute unit; without the next row and the gains in registers 64); rows of 1365 or 5461, at any two bytes, 3.7 to 4.3 TB/s; float32 4.2 to 6.3.
template <bool F32, int TPR, int PK, int GROUPS>
__global__ __launch_bounds__(TPR* GROUPS) void forward_kernel(const void* X, Rows q, Affine p, void* Y, float* stats) {
  __shared__ float2 sh[GROUPS * TPR / 64];
  const int sub = threadIdx.x / TPR, tid = threadIdx.x % TPR;
  const float inv = 1.f / q.d;
  typedef Eight<F32> E8;
  typedef Place<TPR> At;
  float w[PK][8], b[PK][8];
#pragma unroll
  for (int k = 0; k < PK; k++) {
    const At at(k, tid, q.d);
    affine_values(p.w, p.f32, at.at, at.at + 8, w[k], 1.f);
    affine_values(p.b, p.f32, at.at, at.at + 8, b[k], 0.f);
  }
  const int64_t step = (int64_t)gridDim.x * GROUPS;
  typename E8::type raw[PK];
  auto fetch = [&](int64_t row) {
#pragma unroll
    for (int k = 0; k < PK; k++) raw[k] = E8::load(X, row * q.ldx + At(k, tid, q.d).at);
  };
  int64_t row = (int64_t)blockIdx.x * GROUPS + sub;
  if (row < q.n) fetch(row);
  for (int64_t first = (int64_t)blockIdx.x * GROUPS; first < q.n; first += step, row += step) {      // (all rows of a workgroup together: they share barriers)
    float x[PK][8];
#pragma unroll
    for (int k = 0; k < PK; k++) E8::values(raw[k], x[k]);
    if (row + step < q.n) fetch(row + step);
    float s = 0.f, s2 = 0.f;
#pragma unroll
    for (int k = 0; k < PK; k++) {
      const At at(k, tid, q.d);
#pragma unroll
      for (int e = 0; e < 8; e++) s += e >= at.skip ? x[k][e] : 0.f;
    }
    sum2<TPR, GROUPS>(s, s2, sh, sub, tid);
    const float mean = s * inv;
    s = s2 = 0.f;
#pragma unroll
    for (int k = 0; k < PK; k++) {
      const At at(k, tid, q.d);
#pragma unroll
      for (int e = 0; e < 8; e++) {
        x[k][e] -= mean;
        const float c = e >= at.skip ? x[k][e] : 0.f;
        s += c;
        s2 = fmaf(c, c, s2);
      }
    }
    sum2<TPR, GROUPS>(s, s2, sh, sub, tid);
    const float rest = s * inv, rstd = rstd_of(fmaf(s2, inv, -rest * rest), p.eps);
    if (row < q.n) {
      if (stats && tid == 0) { stats[2 * row] = mean + rest; stats[2 * row + 1] = rstd; }
#pragma unroll
      for (int k = 0; k < PK; k++) {
        const At at(k, tid, q.d);
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; e++) y[e] = fmaf((x[k][e] - rest) * rstd, w[k][e], b[k][e]);
        if (at.in) E8::store(Y, row * q.ldy + at.at, y);
      }
    }
  }
}

// Backward: with h = (x - mean) rstd and g = dy w,  dx = rstd (g - mean g - h mean(g h)),  dw = sum over rows of dy h,  db = sum of dy.
// A thread has the same columns in every row that it takes, so the sums over rows stay in its registers; a workgroup's rows are added in order through LDS and go
// to `part` ([workgroup][dw, db][d]), which a second launch adds in order.  Bound by reading X and dY and writing dX: bf16, both launches, 16384 x 2048 38 us (5.3 TB/s), 8192 x 7168 74
// us (4.7), 100000 x 64 14 us (2.7), 4096 x 14336 100 us (3.5; with the next row and the gain in registers 158); float32 4.1 to 5.6.  512 workgroups, with twice the parts: 80 us of 74.
// A few registers do not fit and are kept in memory: 4 of 640 and 12 of 768 threads in float32, 4 of 1024 in both types.
template <bool F32, int TPR, int PK, int GROUPS>
__global__ __launch_bounds__(TPR* GROUPS) void backward_kernel(const void* X, const void* dY, Rows q, int64_t lddy, int64_t lddx, const void* weight, int w_f32,
                                                               const float* __restrict__ stats, void* dX, float* part) {
  __shared__ float2 sh[GROUPS * TPR / 64];
  // Rows of fewer threads than a wave's are added within it first
  constexpr int SUBS = TPR < 64 ? 64 / TPR : 1, PARTS_IN = GROUPS / SUBS;
  constexpr bool HOLD = TPR <= 768;      // the gain stays in registers, and so does the next row; of more threads each has 128 of them
  __shared__ float cols[PARTS_IN > 1 ? 2 * TPR * PK * 8 : 1];
  const int sub = threadIdx.x / TPR, tid = threadIdx.x % TPR;
  const float inv = 1.f / q.d;
  typedef Eight<F32> E8;
  typedef Place<TPR> At;
  float w[HOLD ? PK : 1][8], aw[PK][8], ab[PK][8];
#pragma unroll
  for (int k = 0; k < PK; k++) {
    const At at(k, tid, q.d);
    if constexpr (HOLD) affine_values(weight, w_f32, at.at, at.at + 8, w[k], 1.f);
#pragma unroll
    for (int e = 0; e < 8; e++) aw[k][e] = ab[k][e] = 0.f;
  }
  const int64_t step = (int64_t)gridDim.x * GROUPS;
  typename E8::type rx[PK], ry[PK];
  float2 st{0.f, 0.f};
  auto fetch = [&](int64_t row) {
    st = float2{stats[2 * row], stats[2 * row + 1]};
#pragma unroll
    for (int k = 0; k < PK; k++) {
      rx[k] = E8::load(X, row * q.ldx + At(k, tid, q.d).at);
      ry[k] = E8::load(dY, row * lddy + At(k, tid, q.d).at);
    }
  };
  int64_t row = (int64_t)blockIdx.x * GROUPS + sub;
  if (HOLD && row < q.n) fetch(row);
  for (int64_t first = (int64_t)blockIdx.x * GROUPS; first < q.n; first += step, row += step) {
    const bool mine = row < q.n;
    if (!HOLD && mine) fetch(row);
    float h[PK][8], g[PK][8], s = 0.f, s2 = 0.f;
    const float mean = st.x, rstd = st.y;
#pragma unroll
    for (int k = 0; k < PK; k++) {
      const At at(k, tid, q.d);
      E8::values(rx[k], h[k]);
      E8::values(ry[k], g[k]);
      if constexpr (!HOLD) affine_values(weight, w_f32, at.at, at.at + 8, w[0], 1.f);
#pragma unroll
      for (int e = 0; e < 8; e++) {
        h[k][e] = (h[k][e] - mean) * rstd;
        if (mine) {
          aw[k][e] = fmaf(g[k][e], h[k][e], aw[k][e]);
          ab[k][e] += g[k][e];
        }
        g[k][e] *= w[HOLD ? k : 0][e];
        s += e >= at.skip ? g[k][e] : 0.f;
        s2 = e >= at.skip ? fmaf(g[k][e], h[k][e], s2) : s2;
      }
    }
    if (HOLD && row + step < q.n) fetch(row + step);
    if (!dX) continue;
    sum2<TPR, GROUPS>(s, s2, sh, sub, tid);
    if (mine) {
      s *= inv;
      s2 *= inv;
#pragma unroll
      for (int k = 0; k < PK; k++) {
        const At at(k, tid, q.d);
        float dx[8];
#pragma unroll
        for (int e = 0; e < 8; e++) dx[e] = rstd * fmaf(-h[k][e], s2, g[k][e] - s);
        if (at.in) E8::store(dX, row * lddx + at.at, dx);
      }
    }
  }
  if (!part) return;
  if constexpr (SUBS > 1) {
#pragma unroll
    for (int o = TPR; o < 64; o <<= 1)
#pragma unroll
      for (int k = 0; k < PK; k++)
#pragma unroll
        for (int e = 0; e < 8; e++) { aw[k][e] += __shfl_xor(aw[k][e], o, 64); ab[k][e] += __shfl_xor(ab[k][e], o, 64); }
  }
  const bool speaks = sub % SUBS == 0;      // for its wave's rows
  if constexpr (PARTS_IN > 1) {
    for (int k0 = 0; k0 < PARTS_IN - 1; k0++) {
      if (sub / SUBS == k0 && speaks) {
#pragma unroll
        for (int k = 0; k < PK; k++)
#pragma unroll
          for (int e = 0; e < 8; e++) {
            float* c = cols + ((k * 8 + e) * 2) * TPR + tid;      // (neighbouring threads in neighbouring words)
            c[0] = k0 ? c[0] + aw[k][e] : aw[k][e];
            c[TPR] = k0 ? c[TPR] + ab[k][e] : ab[k][e];
          }
      }
      __syncthreads();
    }
    if (sub / SUBS != PARTS_IN - 1 || !speaks) return;
#pragma unroll
    for (int k = 0; k < PK; k++)
#pragma unroll
      for (int e = 0; e < 8; e++) {
        const float* c = cols + ((k * 8 + e) * 2) * TPR + tid;
        aw[k][e] = c[0] + aw[k][e];
        ab[k][e] = c[TPR] + ab[k][e];
      }
  }
  float* out = part + (int64_t)blockIdx.x * 2 * q.d;
#pragma unroll
  for (int k = 0; k < PK; k++) {
    const At at(k, tid, q.d);
    if (at.in) {
      put_f32(out + at.at, aw[k], 8);
      put_f32(out + q.d + at.at, ab[k], 8);
    }
  }
}

// Long rows, a workgroup each.
template <bool F32>
__global__ __launch_bounds__(1024) void long_forward_kernel(const void* X, Rows q, Affine p, void* Y, float* stats) {
  __shared__ float2 sh[16];
  typedef Eight<F32> E8;
  const int tid = threadIdx.x;
  const float inv = 1.f / q.d;
  for (int64_t row = blockIdx.x; row < q.n; row += gridDim.x) {
    float s = 0.f, s2 = 0.f, x[8];
    auto each = [&](auto f) {
      for (int64_t at = tid * 8; at < q.d; at += 1024 * 8) {
        E8::values(E8::load(X, row * q.ldx + at, q.d - at), x);
        f((int)at);
      }
    };
    each([&](int) {
      float t = 0.f;
#pragma unroll
      for (int e = 0; e < 8; e++) t += x[e];
      s += t;
    });
    sum2<1024, 1>(s, s2, sh, 0, tid);
    const float mean = s * inv;
    s = s2 = 0.f;
    each([&](int at) {
      float t = 0.f, t2 = 0.f;
#pragma unroll
      for (int e = 0; e < 8; e++) {
        const float c = at + e < q.d ? x[e] - mean : 0.f;
        t += c;
        t2 = fmaf(c, c, t2);
      }
      s += t;
      s2 += t2;
    });
    sum2<1024, 1>(s, s2, sh, 0, tid);
    const float rest = s * inv, rstd = rstd_of(fmaf(s2, inv, -rest * rest), p.eps);
    if (stats && tid == 0) { stats[2 * row] = mean + rest; stats[2 * row + 1] = rstd; }
    each([&](int at) {
      float w[8], b[8];
      affine_values(p.w, p.f32, at, q.d, w, 1.f);
      affine_values(p.b, p.f32, at, q.d, b, 0.f);
#pragma unroll
      for (int e = 0; e < 8; e++) x[e] = fmaf((x[e] - mean - rest) * rstd, w[e], b[e]);
      E8::store(Y, row * q.ldy + at, x, q.d - at);
    });
  }
}
template <bool F32>
__global__ __launch_bounds__(1024) void long_backward_kernel(const void* X, const void* dY, Rows q, int64_t lddy, int64_t lddx, const void* weight, int w_f32,
                                                             const float* __restrict__ stats, void* dX) {
  __shared__ float2 sh[16];
  typedef Eight<F32> E8;
  const int tid = threadIdx.x;
  const float inv = 1.f / q.d;
  for (int64_t row = blockIdx.x; row < q.n; row += gridDim.x) {
    const float mean = stats[2 * row], rstd = stats[2 * row + 1];
    float s = 0.f, s2 = 0.f, h[8], g[8], w[8];
    auto each = [&](auto f) {
      for (int64_t at = tid * 8; at < q.d; at += 1024 * 8) {
        E8::values(E8::load(X, row * q.ldx + at, q.d - at), h);
        E8::values(E8::load(dY, row * lddy + at, q.d - at), g);
        affine_values(weight, w_f32, (int)at, q.d, w, 1.f);
#pragma unroll
        for (int e = 0; e < 8; e++) {
          const bool in = at + e < q.d;
          h[e] = in ? (h[e] - mean) * rstd : 0.f;
          g[e] = in ? g[e] * w[e] : 0.f;
        }
        f((int)at);
      }
    };
    each([&](int) {
      float t = 0.f, t2 = 0.f;
#pragma unroll
      for (int e = 0; e < 8; e++) { t += g[e]; t2 = fmaf(g[e], h[e], t2); }
      s += t;
      s2 += t2;
    });
    sum2<1024, 1>(s, s2, sh, 0, tid);
    s *= inv;
    s2 *= inv;
    each([&](int at) {
#pragma unroll
      for (int e = 0; e < 8; e++) g[e] = rstd * fmaf(-h[e], s2, g[e] - s);
      E8::store(dX, row * lddx + at, g, q.d - at);
    });
  }
}
// dw and db of long rows: 2048 columns of a part of the rows (blockIdx.y) per workgroup.  (Before the kernel above, which may write dX over dY or X.)
template <bool F32>
__global__ __launch_bounds__(256) void long_columns_kernel(const void* X, const void* dY, Rows q, int64_t lddy, const float* __restrict__ stats, float* part) {
  typedef Eight<F32> E8;
  const int64_t at = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
  if (at >= q.d) return;
  float aw[8] = {}, ab[8] = {}, h[8], g[8];
  for (int64_t row = blockIdx.y; row < q.n; row += gridDim.y) {
    const float mean = stats[2 * row], rstd = stats[2 * row + 1];
    E8::values(E8::load(X, row * q.ldx + at, q.d - at), h);
    E8::values(E8::load(dY, row * lddy + at, q.d - at), g);
#pragma unroll
    for (int e = 0; e < 8; e++) { aw[e] = fmaf(g[e], (h[e] - mean) * rstd, aw[e]); ab[e] += g[e]; }
  }
  float* out = part + (int64_t)blockIdx.y * 2 * q.d + at;
  const int most = (int)(q.d - at < 8 ? q.d - at : 8);
  put_f32(out, aw, most);
  put_f32(out + q.d, ab, most);
}

// The parts of dw and db added: 64 columns per workgroup, an eighth of the parts per thread, in order (256 parts of 7168: 4.8 us).
__global__ __launch_bounds__(512) void join_columns_kernel(const float* __restrict__ part, int parts, int64_t d, void* dw, void* db, int f32) {
  __shared__ float sh[8][64];
  const int slice = threadIdx.x >> 6, per = (parts + 7) / 8, last = min(parts, (slice + 1) * per);
  for (int64_t base = (int64_t)blockIdx.x * 64; base < 2 * d; base += (int64_t)gridDim.x * 64) {
    const int64_t col = base + (threadIdx.x & 63);      // of dw, then of db
    float s = 0.f;
    if (col < 2 * d) {
#pragma unroll 8
      for (int p = slice * per; p < last; p++) s += part[(int64_t)p * 2 * d + col];
    }
    __syncthreads();
    sh[slice][threadIdx.x & 63] = s;
    __syncthreads();
    if (slice > 0 || col >= 2 * d) continue;
#pragma unroll
    for (int k = 1; k < 8; k++) s += sh[k][threadIdx.x];
    void* out = col < d ? dw : db;
    if (!out) continue;
    const int64_t at = col < d ? col : col - d;
    if (f32) reinterpret_cast<float*>(out)[at] = s;
    else reinterpret_cast<uint16_t*>(out)[at] = bf16_nearest(s);
  }
}

constexpr int FORWARD_BLOCKS = 2048, PARTS = 256;
// The shape of a row: threads, packets of each, and the rows that a workgroup takes together forward and backward.  Few threads beside what the row needs, since the vector units work for every one
// of them: bf16 20000 x 6144 in 384 threads 108 us and backward 136, in 512 118 and 145; 8192 x 9216 in 640 threads 84 and 105, in 1024 114 and 144 (float32 118 and 184, 138 and 196).  Not
// kept, within 3 % or slower: 192 threads of one packet for 1365 columns, 448 for 7168, 896 for 14336.
template <int TPR_, int PK_, int FORWARD_, int BACKWARD_> struct Shape { static constexpr int TPR = TPR_, PK = PK_, FORWARD = FORWARD_, BACKWARD = BACKWARD_; };
template <class F>
void with_shape(int64_t d, F f) {
  if (d <= 64) f(Shape<8, 1, 32, 64>{});
  else if (d <= 128) f(Shape<16, 1, 16, 32>{});
  else if (d <= 256) f(Shape<32, 1, 8, 16>{});
  else if (d <= 512) f(Shape<64, 1, 4, 8>{});
  else if (d <= 1024) f(Shape<64, 2, 4, 8>{});
  else if (d <= 2048) f(Shape<128, 2, 2, 4>{});
  else if (d <= 4096) f(Shape<256, 2, 1, 2>{});
  else if (d <= 320 * 16) f(Shape<320, 2, 1, 1>{});
  else if (d <= 384 * 16) f(Shape<384, 2, 1, 1>{});
  else if (d <= 8192) f(Shape<512, 2, 1, 1>{});
  else if (d <= 640 * 16) f(Shape<640, 2, 1, 1>{});
  else if (d <= 768 * 16) f(Shape<768, 2, 1, 1>{});
  else f(Shape<1024, 2, 1, 1>{});
}
bool in_registers(int64_t d) { return d >= 8 && d <= LONGEST; }
int groups_of(int64_t d) {
  int groups = 1;
  if (in_registers(d)) with_shape(d, [&](auto shape) { groups = decltype(shape)::BACKWARD; });
  return groups;
}
int parts_of(int64_t n, int64_t d) {
  const int64_t groups = groups_of(d), blocks = (n + groups - 1) / groups;
  return (int)(blocks < 1 ? 1 : blocks > PARTS ? PARTS : blocks);
}

template <bool F32, int TPR, int PK, int GROUPS>
void forward(const void* X, const Rows& q, const Affine& p, void* Y, float* stats, hipStream_t s) {
  const int64_t blocks = (q.n + GROUPS - 1) / GROUPS;
  hipLaunchKernelGGL((forward_kernel<F32, TPR, PK, GROUPS>), dim3((unsigned)(blocks < FORWARD_BLOCKS ? blocks : FORWARD_BLOCKS)), dim3(TPR * GROUPS), 0, s, X, q, p, Y, stats);
}
template <bool F32>
void forward_of(const void* X, const Rows& q, const Affine& p, void* Y, float* stats, hipStream_t s) {
  if (!in_registers(q.d))
    hipLaunchKernelGGL(long_forward_kernel<F32>, dim3((unsigned)(q.n < FORWARD_BLOCKS ? q.n : FORWARD_BLOCKS)), dim3(1024), 0, s, X, q, p, Y, stats);
  else
    with_shape(q.d, [&](auto shape) { forward<F32, decltype(shape)::TPR, decltype(shape)::PK, decltype(shape)::FORWARD>(X, q, p, Y, stats, s); });
}
struct Back { const void *X, *dY; Rows q; int64_t lddy, lddx; const void* w; int w_f32; const float* stats; void* dX; float* part; int parts; };
template <bool F32, int TPR, int PK, int GROUPS>
void backward(const Back& a, hipStream_t s) {
  hipLaunchKernelGGL((backward_kernel<F32, TPR, PK, GROUPS>), dim3((unsigned)a.parts), dim3(TPR * GROUPS), 0, s, a.X, a.dY, a.q, a.lddy, a.lddx, a.w, a.w_f32, a.stats, a.dX,
                     a.part);
}
template <bool F32>
void backward_of(const Back& a, hipStream_t s) {
  const int64_t d = a.q.d;
  if (in_registers(d)) {
    with_shape(d, [&](auto shape) { backward<F32, decltype(shape)::TPR, decltype(shape)::PK, decltype(shape)::BACKWARD>(a, s); });
    return;
  }
  if (a.part) hipLaunchKernelGGL(long_columns_kernel<F32>, dim3((unsigned)((d + 2047) / 2048), (unsigned)a.parts), dim3(256), 0, s, a.X, a.dY, a.q, a.lddy, a.stats, a.part);
  if (a.dX) hipLaunchKernelGGL(long_backward_kernel<F32>, dim3((unsigned)(a.q.n < FORWARD_BLOCKS ? a.q.n : FORWARD_BLOCKS)), dim3(1024), 0, s, a.X, a.dY, a.q, a.lddy, a.lddx,
                               a.w, a.w_f32, a.stats, a.dX);
}

bool misaligned(const void* p, int32_t dtype) { return (uintptr_t)p % (dtype == OSSCAR_F32 ? 4 : 2) != 0; }
const char* bad_rows(int64_t n, int64_t d, int64_t ldx, int32_t dtype, int32_t w_dtype) {
  if (!a_size(n, 0) || !a_size(d, 1)) return "osscar_layernorm: n >= 0 and d must be positive, none above 2^30";
  if (!real_dtype(dtype) || !real_dtype(w_dtype)) return "osscar_layernorm: unknown dtype";
  if (ldx < d) return "osscar_layernorm: leading dimension below the row length";
  return nullptr;
}

}  // namespace

extern "C" osscar_status osscar_layernorm_forward(const void* X_dev, int64_t n, int64_t d, int64_t ldx, int32_t dtype, const void* w_dev, const void* b_dev, int32_t w_dtype,
                                                  float eps, void* Y_dev, int64_t ldy, float* stats_dev, void* hip_stream) {
  const char* bad = bad_rows(n, d, ldx, dtype, w_dtype);
  if (!bad && !(eps > 0.f && eps < INFINITY)) bad = "osscar_layernorm_forward: eps must be positive";
  if (!bad && ldy < d) bad = "osscar_layernorm_forward: leading dimension below the row length";
  if (!bad && n > 0 && (!X_dev || !Y_dev)) bad = "osscar_layernorm_forward: NULL pointer";
  if (!bad && (misaligned(X_dev, dtype) || misaligned(Y_dev, dtype) || misaligned(w_dev, w_dtype) || misaligned(b_dev, w_dtype) || misaligned(stats_dev, OSSCAR_F32)))
    bad = "osscar_layernorm_forward: a buffer is not aligned to its elements";
  if (!bad && X_dev == Y_dev && ldx != ldy && n > 1) bad = "osscar_layernorm_forward: in place, both leading dimensions are the same";
  if (bad) return refuse_call(OSSCAR_EINVAL, bad);
  if (n == 0) return OSSCAR_OK;
  hipStream_t s = reinterpret_cast<hipStream_t>(hip_stream);
  const Rows q{n, (int)d, ldx, ldy};
  const Affine p{w_dev, b_dev, w_dtype == OSSCAR_F32, eps};
  if (dtype == OSSCAR_F32) forward_of<true>(X_dev, q, p, Y_dev, stats_dev, s);
  else forward_of<false>(X_dev, q, p, Y_dev, stats_dev, s);
  return launched();
}

extern "C" size_t osscar_layernorm_workspace_bytes(int64_t n, int64_t d) {
  if (!a_size(n, 0) || !a_size(d, 1)) return 0;
  Carve c(nullptr);
  c.take((size_t)parts_of(n, d) * 2 * d * 4);
  return c.used + 256;
}

extern "C" osscar_status osscar_layernorm_backward(const void* X_dev, int64_t n, int64_t d, int64_t ldx, int32_t dtype, const void* w_dev, int32_t w_dtype,
                                                   const void* dY_dev, int64_t lddy, const float* stats_dev, void* dX_dev, int64_t lddx, void* dw_dev, void* db_dev,
                                                   int32_t dw_dtype, void* workspace_dev, size_t workspace_bytes, void* hip_stream) {
  const char* bad = bad_rows(n, d, ldx, dtype, w_dtype);
  const bool sums = dw_dev || db_dev;
  if (!bad && (lddy < d || (dX_dev && lddx < d))) bad = "osscar_layernorm_backward: leading dimension below the row length";
  if (!bad && sums && !real_dtype(dw_dtype)) bad = "osscar_layernorm_backward: unknown dtype";
  if (!bad && n > 0 && (!X_dev || !dY_dev || !stats_dev)) bad = "osscar_layernorm_backward: NULL pointer";
  if (!bad && (misaligned(X_dev, dtype) || misaligned(dY_dev, dtype) || misaligned(dX_dev, dtype) || misaligned(w_dev, w_dtype) || misaligned(stats_dev, OSSCAR_F32) ||
               (sums && (misaligned(dw_dev, dw_dtype) || misaligned(db_dev, dw_dtype)))))
    bad = "osscar_layernorm_backward: a buffer is not aligned to its elements";
  if (!bad && n > 1 && ((dX_dev && dX_dev == X_dev && lddx != ldx) || (dX_dev && dX_dev == dY_dev && lddx != lddy)))
    bad = "osscar_layernorm_backward: in place, both leading dimensions are the same";
  if (!bad && ((uintptr_t)workspace_dev & 255)) bad = "osscar_layernorm_backward: the workspace must begin at a 256-byte boundary";
  if (bad) return refuse_call(OSSCAR_EINVAL, bad);
  if (!sums && (n == 0 || !dX_dev)) return OSSCAR_OK;
  hipStream_t s = reinterpret_cast<hipStream_t>(hip_stream);
  const int parts = parts_of(n, d);
  Carve c(workspace_dev);
  float* part = sums ? reinterpret_cast<float*>(c.take((size_t)parts * 2 * d * 4)) : nullptr;
  if (sums && (!workspace_dev || c.used > workspace_bytes)) return refuse_call(OSSCAR_ENOMEM, "osscar_layernorm_backward: workspace too small");
  const Back a{X_dev, dY_dev, Rows{n, (int)d, ldx, 0}, lddy, lddx, w_dev, w_dtype == OSSCAR_F32, stats_dev, dX_dev, part, parts};
  if (n > 0) {
    if (dtype == OSSCAR_F32) backward_of<true>(a, s);
    else backward_of<false>(a, s);
  }
  // (no rows: no parts, and the sums are zero)
  if (sums) hipLaunchKernelGGL(join_columns_kernel, dim3((unsigned)((2 * d + 63) / 64 < 1 << 20 ? (2 * d + 63) / 64 : 1 << 20)), dim3(512), 0, s, part, n > 0 ? parts : 0, d, dw_dev, db_dev, dw_dtype == OSSCAR_F32);
  return launched();
}
