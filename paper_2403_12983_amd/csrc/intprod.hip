// Products in 8-bit integers with a scale per token and per output channel, and the quantisation of both sides: s_i = max_k |x_ik| / 127, q_ik = rint(x_ik /
// s_i), y_ij = s_i w_j sum_k q_ik Q_jk (+ b_j), the sums exact in int32.  14336 x 7168 with given digits: one row 19 us (5.4 TB/s, thin.h), 64 rows 28 us, 8192
// rows 0.66 ms (2.55 POP/s, tile.h; the library's largest product 2.5).
#include "ops.h"
#include "thin.h"
#include "tile.h"

using namespace osscar;
using namespace osscar::tile;

namespace {

// The scale of a maximum (given as the bits of a non-negative float, which order as the floats do, NaN above all), and a value in it.
__device__ __forceinline__ float scale_of(uint32_t most) { return __uint_as_float(most) / 127.f; }
__device__ __forceinline__ float usable(float s) { return s > 0.f && s < INFINITY ? s : 0.f; }      // else all digits are 0, and s itself makes the result NaN
__device__ __forceinline__ int digit(float x, float s) { return s > 0.f ? (int)fminf(fmaxf(rintf(x / s), -127.f), 127.f) : 0; }
__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

typedef int8_t s8x8 __attribute__((ext_vector_type(8)));

// One row by T threads: its digits, zeros from d1 to ldq, and its scale; sh: T / 64 words.  x (1 / s) is within 3 2^-24 127 = 2.3e-5 of the rounded quotient x
// / s, so that both have the same nearest integer unless one lies closer than that to a half; only there, and where 1 / s might be no normal number, is divided
// (everywhere: 97 us for 8192 x 14336 bf16; so 91, 3.9 TB/s).
template <int T>
__device__ __forceinline__ float row_digits(const void* __restrict__ X, int64_t at, int f32, int d1, int8_t* __restrict__ q8, int ldq, uint32_t* sh) {
  uint32_t most = 0;
  for (int k = threadIdx.x * 8; k < d1; k += T * 8) {
    float v[8];
    get_values(X, at + k, f32, v, d1 - k);
#pragma unroll
    for (int e = 0; e < 8; e++) most = max(most, magnitude(v[e]));
  }
  for (int o = 32; o > 0; o >>= 1) most = max(most, (uint32_t)__shfl_xor((int)most, o, 64));
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = most;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < T / 64; w++) most = max(most, sh[w]);
  const float s = scale_of(most), u = usable(s), r = 1.f / u;
  const bool quick = u > 1e-30f && u < 1e30f;
  for (int k = threadIdx.x * 8; k < ldq; k += T * 8) {
    float v[8];
    get_values(X, at + k, f32, v, d1 - k);      // (zeros past d1)
    s8x8 w;
    float far = quick ? 0.f : 1.f;
#pragma unroll
    for (int e = 0; e < 8; e++) {
      const float y = v[e] * r, q = rintf(y);
      far = fmaxf(far, fabsf(y - q));
      w[e] = (int8_t)q;
    }
    if (far > 0.49996f)
#pragma unroll
      for (int e = 0; e < 8; e++) w[e] = (int8_t)(k + e < d1 ? digit(v[e], u) : 0);
    *reinterpret_cast<s8x8*>(q8 + k) = w;
  }
  return s;
}
// One row per workgroup, read twice (the second time from cache).  Bound by reading X and writing Xq; few rows: by the latency of the steps, so that they get
// 1024 threads each.  Weights m x d1 come here too, once per layer: 7168 rows of 14336 bf16 77 us (4.0 TB/s), float32 139 us.
template <int T>
__global__ __launch_bounds__(T) void int_rows_kernel(const void* __restrict__ X, int f32, int d1, int64_t ldx, int8_t* __restrict__ Xq, int64_t ldq,
                                                       float* __restrict__ scale) {
  __shared__ uint32_t sh[T / 64];
  const int64_t row = blockIdx.x;
  const float s = row_digits<T>(X, row * ldx, f32, d1, Xq + row * ldq, (int)ldq, sh);
  if (threadIdx.x == 0) scale[row] = s;
}
// copies digits to rows of ldq, zeros past d1
__global__ __launch_bounds__(256) void int_copy_kernel(const int8_t* __restrict__ X, int64_t n, int d1, int64_t ldx, int8_t* __restrict__ Xq, int64_t ldq) {
  for (int64_t i = blockIdx.x * (int64_t)256 + threadIdx.x; i < n * ldq; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / ldq;
    const int k = (int)(i - r * ldq);
    Xq[i] = k < d1 ? X[r * ldx + k] : (int8_t)0;
  }
}
// Columns of W (d1 x m): the maxima, 64 rows per workgroup and 256 columns, joined by an atomic maximum (the order does not matter).  W is read twice, a number
// per thread: 14336 x 7168 bf16 233 us for all four launches (2.2 TB/s), float32 310 us, once per layer.
__global__ void int_zero_kernel(uint32_t* p, int n) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i < n) p[i] = 0u;
}
__global__ __launch_bounds__(256) void int_column_max_kernel(const void* __restrict__ W, int f32, int d1, int m, int64_t ldw, uint32_t* __restrict__ most) {
  const int j = blockIdx.x * 256 + threadIdx.x, k0 = blockIdx.y * 64, k1 = min(d1, k0 + 64);
  if (j >= m) return;
  uint32_t v = 0;
  for (int k = k0; k < k1; k++) {
    const int64_t at = (int64_t)k * ldw + j;
    v = max(v, magnitude(f32 ? reinterpret_cast<const float*>(W)[at] : bf16_value(reinterpret_cast<const uint16_t*>(W)[at])));
  }
  atomicMax(most + j, v);
}
__global__ void int_scales_kernel(uint32_t* p, int n) {      // maxima become scales
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i < n) p[i] = __float_as_uint(scale_of(p[i]));
}
// 64 x 64 blocks turned over in LDS
__global__ __launch_bounds__(256) void int_columns_kernel(const void* __restrict__ W, int f32, int d1, int m, int64_t ldw, const float* __restrict__ scale,
                                                          int8_t* __restrict__ Wq, int64_t ldq) {
  __shared__ int8_t T[64][68];
  const int k0 = blockIdx.x * 64, j0 = blockIdx.y * 64, c = threadIdx.x & 63, r = threadIdx.x >> 6;
  const float u = j0 + c < m ? usable(scale[j0 + c]) : 0.f;
  for (int k = r; k < 64; k += 4) {
    float x = 0.f;
    if (k0 + k < d1 && j0 + c < m) {
      const int64_t at = (int64_t)(k0 + k) * ldw + j0 + c;
      x = f32 ? reinterpret_cast<const float*>(W)[at] : bf16_value(reinterpret_cast<const uint16_t*>(W)[at]);
    }
    T[c][k] = (int8_t)digit(x, u);
  }
  __syncthreads();
  for (int j = r; j < 64; j += 4)
    if (j0 + j < m && k0 + c < ldq) Wq[(int64_t)(j0 + j) * ldq + k0 + c] = T[j][c];
}

struct IntOut {
  const float *xs, *ws, *bias; void* Y; int64_t ldy; int f32;
  template <class F>
  __device__ __forceinline__ void each(F f) const {
    f([&](int m, int n, const int (&v)[1][8], int N) {
      const float s = xs[m];
      float y[8];
#pragma unroll
      for (int c = 0; c < 8; c++) {
        const int j = min(n + c, N - 1);
        y[c] = (float)v[0][c] * s * ws[j];
        if (bias) y[c] += bias[j];
      }
      if (f32) put_f32(reinterpret_cast<float*>(Y) + (int64_t)m * ldy + n, y, N - n);
      else put_bf16(reinterpret_cast<uint16_t*>(Y) + (int64_t)m * ldy + n, y, N - n);
    });
  }
  template <class F>
  __device__ __forceinline__ void one(F f) const {
    f([&](int m, int n, const int (&v)[1], int) {
      float y = (float)v[0] * xs[m] * ws[n];
      if (bias) y += bias[n];
      if (f32) reinterpret_cast<float*>(Y)[(int64_t)m * ldy + n] = y;
      else reinterpret_cast<uint16_t*>(Y)[(int64_t)m * ldy + n] = bf16_nearest(y);
    });
  }
};
typedef Shape<2, 2, 8, 8, 1> Big;        // 256 x 256, four waves
typedef Shape<2, 2, 4, 4, 1> Small;      // 128 x 128, four waves

template <class S>
__global__ __launch_bounds__(S::WAVES * 64, 1) void int_product_kernel(const Product<1> p, const IntOut e) {
  product_tile<true, OP_K, OP_K, S>(p, e);
}

template <bool WIDE>
__global__ __launch_bounds__((thin::Wave<OP_K, thin::I8, 1, 1, WIDE>::WAVES) * 64, 1) void int_thin_kernel(const thin::Product<1> p, const IntOut e) {
  thin::product<OP_K, thin::I8, 1, 1, WIDE>(p, e);
}
// The same for one row that is not digits yet: every workgroup makes them for itself, in LDS; scale: where the first one leaves the scale for a join.  Taken
// for rows of up to TOKEN_DIM and no more than two workgroups per compute unit, where it costs less than a launch before (14336 x 7168 21.8 us and 24.5, 2048 x
// 2048 9.9 and 13.2; 32768 x 4096 39 and 35, 7168 x 14336 in 896 workgroups 25 and 23; two rows 26 and 23).
constexpr int TOKEN_DIM = 16384, TOKEN_BLOCKS = 512;
__global__ __launch_bounds__(512, 1) void int_token_kernel(const void* __restrict__ X, int f32, int ldq, float* __restrict__ scale, thin::Product<1> p, IntOut e) {
  static_assert(thin::Wave<OP_K, thin::I8, 1, 1, false>::WAVES == 8, "");
  __shared__ __align__(16) int8_t digits[TOKEN_DIM];
  __shared__ float own;
  __shared__ uint32_t sh[8];
  const float s = row_digits<512>(X, 0, f32, p.K, digits, ldq, sh);
  if (threadIdx.x == 0) {
    own = s;
    if (blockIdx.x == 0 && blockIdx.y == 0) *scale = s;
  }
  __syncthreads();
  p.a = reinterpret_cast<const char*>(digits);
  e.xs = &own;
  thin::product<OP_K, thin::I8, 1, 1, false>(p, e);
}
__global__ __launch_bounds__(256) void int_join_kernel(const int* __restrict__ sums, int parts, int M, int N, const IntOut e) {
  tile::join<1>(sums, parts, M, N, e);
}

template <class S, int G>
__global__ __launch_bounds__(256) void int_join_tiles_kernel(const Product<1> p, const IntOut e) { tile::join_tiles<S, int, G>(p, e); }
template <class S>
void launch_join(const Product<1>& p, const IntOut& e, const Deal& d, hipStream_t s) {
  if (d.parts >= JOIN_GROUPS_FROM) hipLaunchKernelGGL((int_join_tiles_kernel<S, 4>), dim3((unsigned)d.join), dim3(256), 0, s, p, e);
  else hipLaunchKernelGGL((int_join_tiles_kernel<S, 1>), dim3((unsigned)d.join), dim3(256), 0, s, p, e);
}

inline int64_t up16(int64_t v) { return (v + 15) / 16 * 16; }
template <class S>
int64_t tiles(int64_t n, int64_t m) { return (n + S::BM - 1) / S::BM * ((m + S::BN - 1) / S::BN); }
Deal deal_of(int64_t n, int64_t d1, int64_t m) { return deal<Big, Small>(n, m, (d1 + STEP_BYTES - 1) / STEP_BYTES, 1); }
bool few_rows(int64_t n) { return n <= 16; }      // (thin.h says why)
bool bad_sizes(int64_t n, int64_t d1, int64_t m) { return !a_size(n, 0) || !a_size(m, 1) || d1 < 1 || d1 > OSSCAR_INT_MAX_DIM || tiles<Small>(n, m) > 0x3FFFFFFF; }
bool launchable_product(int64_t n, int64_t d1, int64_t m) {
  const thin::Deal d = thin::deal<OP_K, thin::I8>(n, m, d1);
  return n == 0 || (few_rows(n) ? launchable(d.blocks, d.threads) : launchable(deal_of(n, d1, m).blocks, 256));
}
bool bad_digits(const void* q, int64_t ldq, int64_t d1) { return !q || (uintptr_t)q % 16 || ldq % 16 || ldq < d1 || ldq > MAX_LD_BYTES; }

void quantise_rows(const void* X, int64_t n, int64_t d1, int64_t ldx, int f32, int8_t* Xq, int64_t ldq, float* scale, hipStream_t s) {
  if (n <= 256) {
    hipLaunchKernelGGL(int_rows_kernel<1024>, dim3((unsigned)n), dim3(1024), 0, s, X, f32, (int)d1, ldx, Xq, ldq, scale);
    return;
  }
  constexpr int64_t LAUNCH = 1 << 23;      // rows: a launch has fewer than 2^32 threads along a dimension
  for (int64_t r = 0; r < n; r += LAUNCH)
    hipLaunchKernelGGL(int_rows_kernel<256>, dim3((unsigned)(n - r < LAUNCH ? n - r : LAUNCH)), dim3(256), 0, s, reinterpret_cast<const char*>(X) + r * ldx * (f32 ? 4 : 2), f32, (int)d1, ldx,
                       Xq + r * ldq, ldq, scale + r);
}

}  // namespace

extern "C" osscar_status osscar_int_rows(const void* X_dev, int64_t n, int64_t d1, int64_t ldx, int32_t x_dtype, int8_t* Xq_dev, int64_t ldq, float* x_scale_dev,
                                         void* hip_stream) {
  if (bad_sizes(n, d1, 1)) return refuse_call(OSSCAR_EINVAL, "osscar_int_rows: n >= 0 and 1 <= d1 <= OSSCAR_INT_MAX_DIM");
  if (!real_dtype(x_dtype)) return refuse_call(OSSCAR_EINVAL, "osscar_int_rows: unknown dtype");
  if (n == 0) return OSSCAR_OK;
  if (!X_dev || ldx < d1 || !x_scale_dev || (uintptr_t)X_dev % (x_dtype == OSSCAR_F32 ? 4 : 2)) return refuse_call(OSSCAR_EINVAL, "osscar_int_rows: NULL or misaligned pointer, or leading dimension below the row length");
  if (bad_digits(Xq_dev, ldq, d1)) return refuse_call(OSSCAR_EINVAL, "osscar_int_rows: Xq begins at a 16-byte boundary and ldq is a multiple of 16");
  quantise_rows(X_dev, n, d1, ldx, x_dtype == OSSCAR_F32, Xq_dev, ldq, x_scale_dev, reinterpret_cast<hipStream_t>(hip_stream));
  return launched();
}

extern "C" osscar_status osscar_int_weights(const void* W_dev, int64_t d1, int64_t m, int64_t ldw, int32_t w_dtype, int32_t rows_out, int8_t* Wq_dev, int64_t ldq,
                                            float* w_scale_dev, void* hip_stream) {
  if (bad_sizes(0, d1, m)) return refuse_call(OSSCAR_EINVAL, "osscar_int_weights: m must be positive and 1 <= d1 <= OSSCAR_INT_MAX_DIM");
  if (!real_dtype(w_dtype)) return refuse_call(OSSCAR_EINVAL, "osscar_int_weights: unknown dtype");
  if (!W_dev || !w_scale_dev || ldw < (rows_out ? d1 : m) || (uintptr_t)W_dev % (w_dtype == OSSCAR_F32 ? 4 : 2))
    return refuse_call(OSSCAR_EINVAL, "osscar_int_weights: NULL or misaligned pointer, or leading dimension below the row length");
  if (bad_digits(Wq_dev, ldq, d1)) return refuse_call(OSSCAR_EINVAL, "osscar_int_weights: Wq begins at a 16-byte boundary and ldq is a multiple of 16");
  hipStream_t s = reinterpret_cast<hipStream_t>(hip_stream);
  const int f32 = w_dtype == OSSCAR_F32;
  if (rows_out) {
    quantise_rows(W_dev, m, d1, ldw, f32, Wq_dev, ldq, w_scale_dev, s);
  } else {
    uint32_t* most = reinterpret_cast<uint32_t*>(w_scale_dev);
    const unsigned mb = (unsigned)((m + 255) / 256);
    hipLaunchKernelGGL(int_zero_kernel, dim3(mb), dim3(256), 0, s, most, (int)m);
    hipLaunchKernelGGL(int_column_max_kernel, dim3(mb, (unsigned)((d1 + 63) / 64)), dim3(256), 0, s, W_dev, f32, (int)d1, (int)m, ldw, most);
    hipLaunchKernelGGL(int_scales_kernel, dim3(mb), dim3(256), 0, s, most, (int)m);
    for (int64_t j0 = 0; j0 < m; j0 += (int64_t)64 * 65535) {      // (the grid's second dimension ends at 65535)
      const int64_t part = m - j0 < (int64_t)64 * 65535 ? m - j0 : (int64_t)64 * 65535;
      hipLaunchKernelGGL(int_columns_kernel, dim3((unsigned)((ldq + 63) / 64), (unsigned)((part + 63) / 64)), dim3(256), 0, s,
                         reinterpret_cast<const char*>(W_dev) + j0 * (f32 ? 4 : 2), f32, (int)d1, (int)part, ldw, w_scale_dev + j0, Wq_dev + j0 * ldq, ldq);
    }
  }
  return launched();
}

extern "C" size_t osscar_int_workspace_bytes(int64_t n, int64_t d1, int64_t m) {
  if (bad_sizes(n, d1, m) || !launchable_product(n, d1, m)) return 0;
  Carve c(nullptr);
  c.take((size_t)n * up16(d1));
  c.take((size_t)n * 4);
  c.take(few_rows(n) ? (size_t)thin::deal<OP_K, thin::I8>(n, m, d1).parts * n * m * 4 : deal_of(n, d1, m).sums);
  return c.used + 256;
}

extern "C" osscar_status osscar_int_product(const void* X_dev, int64_t n, int64_t d1, int64_t ldx, int32_t x_dtype, const float* x_scale_dev, const int8_t* Wq_dev,
                                            int64_t ldq, const float* w_scale_dev, int64_t m, const float* bias_dev, void* Y_dev, int64_t ldy, int32_t y_dtype,
                                            void* workspace_dev, size_t workspace_bytes, void* hip_stream) {
  if (bad_sizes(n, d1, m)) return refuse_call(OSSCAR_EINVAL, "osscar_int_product: n >= 0, m must be positive and 1 <= d1 <= OSSCAR_INT_MAX_DIM");
  if (!launchable_product(n, d1, m)) return refuse_call(OSSCAR_EINVAL, "osscar_int_product: the product of the sizes is too large for one call");
  if ((!real_dtype(x_dtype) && x_dtype != OSSCAR_I8) || !real_dtype(y_dtype)) return refuse_call(OSSCAR_EINVAL, "osscar_int_product: unknown dtype");
  if (n == 0) return OSSCAR_OK;
  const bool given = x_dtype == OSSCAR_I8;
  if (!X_dev || !w_scale_dev || !Y_dev || ldx < d1 || ldy < m || given != (x_scale_dev != nullptr))
    return refuse_call(OSSCAR_EINVAL, "osscar_int_product: NULL pointer, leading dimension below the row length, or x_scale not exactly with 8-bit X");
  if (!given && (uintptr_t)X_dev % (x_dtype == OSSCAR_F32 ? 4 : 2)) return refuse_call(OSSCAR_EINVAL, "osscar_int_product: X is not aligned to its elements");
  if ((uintptr_t)Y_dev % (y_dtype == OSSCAR_F32 ? 4 : 2)) return refuse_call(OSSCAR_EINVAL, "osscar_int_product: Y is not aligned to its elements");
  if (bad_digits(Wq_dev, ldq, d1)) return refuse_call(OSSCAR_EINVAL, "osscar_int_product: Wq begins at a 16-byte boundary and ldq is a multiple of 16");
  if ((uintptr_t)workspace_dev & 255) return refuse_call(OSSCAR_EINVAL, "osscar_int_product: the workspace must begin at a 256-byte boundary");
  hipStream_t s = reinterpret_cast<hipStream_t>(hip_stream);
  const int8_t* xq = reinterpret_cast<const int8_t*>(X_dev);
  const float* xs = x_scale_dev;
  int64_t ldxq = ldx;
  const bool few = few_rows(n);
  Carve c(workspace_dev);
  const thin::Deal thin_deal = thin::deal<OP_K, thin::I8>(n, m, d1);
  const bool token = !given && n == 1 && d1 <= TOKEN_DIM && (int64_t)thin_deal.blocks * thin_deal.parts <= TOKEN_BLOCKS;
  float* scales = nullptr;      // made here
  if (token) {
    xs = scales = reinterpret_cast<float*>(c.take(4));
    if (!workspace_dev || c.used > workspace_bytes) return refuse_call(OSSCAR_ENOMEM, "osscar_int_product: workspace too small");
  } else if (!given || (!few && !operand_fits(X_dev, ldx, d1, 1))) {
    ldxq = up16(d1);
    int8_t* q = reinterpret_cast<int8_t*>(c.take((size_t)n * ldxq));
    float* sc = reinterpret_cast<float*>(c.take((size_t)n * 4));
    if (!workspace_dev || c.used > workspace_bytes) return refuse_call(OSSCAR_ENOMEM, "osscar_int_product: workspace too small");
    if (given) {
      const int64_t g = (n * ldxq + 255) / 256;
      hipLaunchKernelGGL(int_copy_kernel, dim3((unsigned)(g > 8192 ? 8192 : g)), dim3(256), 0, s, xq, n, (int)d1, ldx, q, ldxq);
    } else {
      quantise_rows(X_dev, n, d1, ldx, x_dtype == OSSCAR_F32, q, ldxq, sc, s);
      xs = sc;
    }
    xq = q;
  }
  const IntOut e{xs, w_scale_dev, bias_dev, Y_dev, ldy, y_dtype == OSSCAR_F32};
  if (few) {
    const thin::Deal& d = thin_deal;
    thin::Product<1> t{reinterpret_cast<const char*>(xq), {reinterpret_cast<const char*>(Wq_dev)}, ldxq, ldq, (int)n, (int)m, (int)d1, d.parts, nullptr};
    if (t.parts > 1) {
      t.sums = c.take((size_t)t.parts * n * m * 4);
      if (!workspace_dev || c.used > workspace_bytes) return refuse_call(OSSCAR_ENOMEM, "osscar_int_product: workspace too small");
    }
    const dim3 grid(d.blocks, (unsigned)d.parts), block(512);
    if (token) hipLaunchKernelGGL(int_token_kernel, grid, block, 0, s, X_dev, x_dtype == OSSCAR_F32, (int)up16(d1), scales, t, e);
    else if (d.wide) hipLaunchKernelGGL(int_thin_kernel<true>, grid, block, 0, s, t, e);
    else hipLaunchKernelGGL(int_thin_kernel<false>, grid, block, 0, s, t, e);
    if (t.parts > 1)
      hipLaunchKernelGGL(int_join_kernel, dim3(join_grid(n, m)), dim3(256), 0, s, reinterpret_cast<const int*>(t.sums), t.parts, (int)n, (int)m, e);
    return launched();
  }
  Product<1> p{};
  p.a.p[0] = reinterpret_cast<const char*>(xq); p.a.ldb = ldxq; p.a.rows = (int)n; p.a.cols = (int)up16(d1);
  p.b[0].p[0] = reinterpret_cast<const char*>(Wq_dev); p.b[0].ldb = ldq; p.b[0].rows = (int)m; p.b[0].cols = (int)up16(d1);
  p.nseg = 1; p.k = (int)d1; p.M = (int)n; p.N = (int)m;
  const Deal d = deal_of(n, d1, m);
  p.whole = d.whole;
  p.parts = d.parts;
  if (d.parts > 1) {
    p.sums = c.take(d.sums);
    if (!workspace_dev || c.used > workspace_bytes) return refuse_call(OSSCAR_ENOMEM, "osscar_int_product: workspace too small");
  }
  const dim3 grid(d.blocks);
  if (d.pick == BIG_TILE) hipLaunchKernelGGL(int_product_kernel<Big>, grid, dim3(Big::WAVES * 64), 0, s, p, e);
  else hipLaunchKernelGGL(int_product_kernel<Small>, grid, dim3(Small::WAVES * 64), 0, s, p, e);
  if (d.parts > 1) d.pick == BIG_TILE ? launch_join<Big>(p, e, d, s) : launch_join<Small>(p, e, d, s);
  return launched();
}
