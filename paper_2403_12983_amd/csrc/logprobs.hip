// Log probabilities of given tokens, entropy and largest alternatives from logits, and the gradient.
#include "ops.h"
#include <float.h>

using namespace osscar;

namespace {

constexpr float LOG2E = 1.44269504088896341f, LN2 = 0.69314718055994531f;

// Running state of a row's softmax: the largest logit m so far (raw, at least -FLT_MAX so that differences with it exist), S = sum 2^y and
// A = sum -y 2^y with y = scale log2(e) (l - m) <= 0.  log sum exp = scale m + ln S and entropy = ln S + ln2 A / S: sums of terms
// of one sign.  A row of minus infinities leaves S = 0; NaN and plus infinity make S NaN.
struct Stat { float m, S, A; };
// the largest grows from s.m to m
__device__ __forceinline__ void raise(Stat& s, float m, float c2) {
  const float d = (s.m - m) * c2, e = exp2f(d);      // d <= 0
  s.A = e * (s.A - fmaxf(d, -200.f) * s.S);
  s.S *= e;
  s.m = m;
}
__device__ __forceinline__ void add(Stat& s, float l, float c2) {
  const float y = (l - s.m) * c2, e = exp2f(y);
  s.S += e;
  s.A -= fmaxf(y, -200.f) * e;      // (2^-200 is 0: y = -inf adds nothing)
}
__device__ __forceinline__ void join(Stat& s, Stat o, float c2) {
  const float m = fmaxf(s.m, o.m);
  raise(s, m, c2);
  raise(o, m, c2);
  s.S += o.S;
  s.A += o.A;
}
__device__ __forceinline__ float entropy_of(const Stat& s) { return s.S == 0.f ? 0.f : logf(s.S) + LN2 * (s.A / s.S); }
__device__ __forceinline__ float logp_of(const Stat& s, float l, float scale) { return s.S == 0.f ? -INFINITY : scale * (l - s.m) - logf(s.S); }

// Order of alternatives: larger value first, then lower index; NaN above all, the two zeros equal.
__device__ __forceinline__ uint64_t rank_of(float l, uint32_t v) {
  uint32_t b = __float_as_uint(l + 0.f);
  if (l != l) b = 0x7FC00000u;
  b ^= (b & 0x80000000u) ? 0xFFFFFFFFu : 0x80000000u;
  return (uint64_t)b << 32 | (0xFFFFFFFFu - v);
}
__device__ __forceinline__ uint32_t index_of(uint64_t r) { return 0xFFFFFFFFu - (uint32_t)r; }

__device__ __forceinline__ float logit(const void* p, int f32, int64_t at) {
  return f32 ? reinterpret_cast<const float*>(p)[at] : bf16_value(reinterpret_cast<const uint16_t*>(p)[at]);
}

constexpr int T = 256;

// One row per workgroup.
__global__ __launch_bounds__(T) void logprobs_kernel(const void* __restrict__ logits, int f32, int vocab, int64_t ld, const int64_t* __restrict__ targets, float scale,
                                                     int top, float* __restrict__ logp, float* __restrict__ entropy, float* __restrict__ lse,
                                                     int64_t* __restrict__ top_index, float* __restrict__ top_logp) {
  __shared__ Stat st[T / 64];
  __shared__ uint64_t rk[T / 64];
  const int64_t row = blockIdx.x, base = row * ld;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const float c2 = scale * LOG2E;
  Stat s{-FLT_MAX, 0.f, 0.f};
  for (int v0 = tid * 8; v0 < vocab; v0 += T * 8) {
    float l[8];
    get_values(logits, base + v0, f32, l, vocab - v0);
    const int most = min(8, vocab - v0);
    float m = s.m;
#pragma unroll
    for (int e = 0; e < 8; e++) {
      if (e >= most) l[e] = -INFINITY;
      m = fmaxf(m, l[e]);
    }
    if (m > s.m) raise(s, m, c2);
#pragma unroll
    for (int e = 0; e < 8; e++) add(s, l[e], c2);
  }
  for (int o = 32; o > 0; o >>= 1) join(s, Stat{__shfl_xor(s.m, o, 64), __shfl_xor(s.S, o, 64), __shfl_xor(s.A, o, 64)}, c2);
  if (lane == 0) st[wave] = s;
  __syncthreads();
  s = st[0];
#pragma unroll
  for (int w = 1; w < T / 64; w++) join(s, st[w], c2);
  if (tid == 0) {
    const int64_t t = targets[row];
    logp[row] = t < 0 ? 0.f : (t >= vocab ? NAN : logp_of(s, logit(logits, f32, base + t), scale));
    if (entropy) entropy[row] = entropy_of(s);
    if (lse) { lse[2 * row] = s.m; lse[2 * row + 1] = s.S == 0.f ? -INFINITY : logf(s.S); }
  }
  uint64_t last = ~0ull;
  for (int j = 0; j < top; j++) {
    uint64_t best = 0;
    for (int v = tid; v < vocab; v += T) {
      const uint64_t r = rank_of(logit(logits, f32, base + v), v);
      if (r < last && r > best) best = r;
    }
    for (int o = 32; o > 0; o >>= 1) { const uint64_t x = __shfl_xor((unsigned long long)best, o, 64); best = x > best ? x : best; }
    __syncthreads();
    if (lane == 0) rk[wave] = best;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < T / 64; w++) best = rk[w] > best ? rk[w] : best;
    last = best;
    if (tid == 0) {
      const uint32_t v = index_of(best);
      top_index[row * top + j] = v;
      top_logp[row * top + j] = logp_of(s, logit(logits, f32, base + v), scale);
    }
  }
}

// Gradient.  A workgroup takes CHUNK columns of a row; the few columns that have a term of their own (target, alternatives) are computed by a
// thread each from logits read before the others are written.
constexpr int CHUNK = T * 8 * 4;
__global__ __launch_bounds__(T) void logprobs_backward_kernel(const void* logits, int f32, int vocab, int64_t ld, const int64_t* __restrict__ targets, float scale,
                                                              const float* __restrict__ lse, const float* __restrict__ dlogp, const float* __restrict__ entropy,
                                                              const float* __restrict__ dentropy, int top, const int64_t* __restrict__ top_index,
                                                              const float* __restrict__ dtop, void* out, int64_t ldd) {
  const int64_t row = blockIdx.y;
  const int tid = threadIdx.x, c0 = blockIdx.x * CHUNK, c1 = min(vocab, c0 + CHUNK);
  const float m = lse[2 * row], lnS = lse[2 * row + 1];
  const int64_t t = targets[row];
  float dl = dlogp && t >= 0 ? (t >= vocab ? NAN : dlogp[row]) : 0.f;
  const float dh = dentropy ? dentropy[row] : 0.f, H = dentropy ? entropy[row] : 0.f;
  float w = dl;
  for (int j = 0; j < top; j++) w += dtop[row * top + j];
  const bool empty = lnS == -INFINITY;
  auto grad = [&](float l, float own) {
    const float lp = scale * (l - m) - lnS, p = __expf(lp);
    const float x = p == 0.f ? 0.f : -p * (w + dh * (lp + H));
    return empty ? 0.f : scale * (x + own);
  };
  // this thread's special column: the target (thread 0) or an alternative
  int64_t col = -1;
  if (tid <= top) col = tid == 0 ? (dl == 0.f ? -1 : t) : top_index[row * top + tid - 1];
  float mine = 0.f;
  const bool special = col >= c0 && col < c1;
  if (special) {
    float own = dlogp && col == t ? dl : 0.f;
    for (int j = 0; j < top; j++) own += top_index[row * top + j] == col ? dtop[row * top + j] : 0.f;
    mine = grad(logit(logits, f32, row * ld + col), own);
  }
  __syncthreads();
  for (int v0 = c0 + tid * 8; v0 < c1; v0 += T * 8) {
    float l[8];
    get_values(logits, row * ld + v0, f32, l, vocab - v0);
#pragma unroll
    for (int e = 0; e < 8; e++) l[e] = grad(l[e], 0.f);
    if (f32) put_f32(reinterpret_cast<float*>(out) + row * ldd + v0, l, vocab - v0);
    else put_bf16(reinterpret_cast<uint16_t*>(out) + row * ldd + v0, l, vocab - v0);
  }
  __syncthreads();
  if (special) {
    if (f32) reinterpret_cast<float*>(out)[row * ldd + col] = mine;
    else reinterpret_cast<uint16_t*>(out)[row * ldd + col] = bf16_nearest(mine);
  }
}

const char* bad_logits(const void* logits, int64_t n, int64_t vocab, int64_t ld, int32_t dtype, const int64_t* targets, float scale, int32_t top) {
  if (!a_size(n, 0) || !a_size(vocab, 1)) return "osscar_logprobs: n >= 0 and vocab must be positive, none above 2^30";
  if (!real_dtype(dtype)) return "osscar_logprobs: unknown dtype";
  if (!(scale > 0.f && scale < INFINITY)) return "osscar_logprobs: scale must be positive and finite";
  if (top < 0 || top > OSSCAR_TOP_MAX || top > vocab) return "osscar_logprobs: top is at most OSSCAR_TOP_MAX and at most vocab";
  if (n > 0 && (!logits || !targets || ld < vocab)) return "osscar_logprobs: NULL pointer or leading dimension below the row length";
  if ((uintptr_t)logits % (dtype == OSSCAR_F32 ? 4 : 2)) return "osscar_logprobs: logits are not aligned to their elements";
  return nullptr;
}

}  // namespace

extern "C" size_t osscar_logprobs_workspace_bytes(int64_t n, int64_t vocab, int32_t top) {
  if (!a_size(n, 0) || !a_size(vocab, 1) || top < 0 || top > OSSCAR_TOP_MAX || top > vocab) return 0;
  return 256;
}

extern "C" osscar_status osscar_logprobs(const void* logits_dev, int64_t n, int64_t vocab, int64_t ld, int32_t dtype, const int64_t* targets_dev, float scale,
                                         int32_t top, float* logp_dev, float* entropy_dev, float* lse_dev, int64_t* top_index_dev, float* top_logp_dev,
                                         void* workspace_dev, size_t workspace_bytes, void* hip_stream) {
  const char* bad = bad_logits(logits_dev, n, vocab, ld, dtype, targets_dev, scale, top);
  if (!bad && n > 0 && (!logp_dev || (top > 0 && (!top_index_dev || !top_logp_dev)))) bad = "osscar_logprobs: NULL pointer";
  if (!bad && ((uintptr_t)workspace_dev & 255)) bad = "osscar_logprobs: the workspace must begin at a 256-byte boundary";
  if (bad) return refuse_call(OSSCAR_EINVAL, bad);
  if (n == 0) return OSSCAR_OK;
  (void)workspace_bytes;
  hipStream_t s = reinterpret_cast<hipStream_t>(hip_stream);
  hipLaunchKernelGGL(logprobs_kernel, dim3((unsigned)n), dim3(T), 0, s, logits_dev, dtype == OSSCAR_F32, (int)vocab, ld, targets_dev, scale, top, logp_dev,
                     entropy_dev, lse_dev, top_index_dev, top_logp_dev);
  return launched("osscar_logprobs");
}

extern "C" osscar_status osscar_logprobs_backward(const void* logits_dev, int64_t n, int64_t vocab, int64_t ld, int32_t dtype, const int64_t* targets_dev, float scale,
                                                  const float* lse_dev, const float* dlogp_dev, const float* entropy_dev, const float* dentropy_dev, int32_t top,
                                                  const int64_t* top_index_dev, const float* dtop_dev, void* dlogits_dev, int64_t ldd, void* hip_stream) {
  if (!dtop_dev) top = 0;
  const char* bad = bad_logits(logits_dev, n, vocab, ld, dtype, targets_dev, scale, top);
  if (!bad && n > 0 && (!lse_dev || !dlogits_dev || ldd < vocab || (dentropy_dev && !entropy_dev) || (top > 0 && !top_index_dev)))
    bad = "osscar_logprobs_backward: NULL pointer or leading dimension below the row length";
  if (!bad && (uintptr_t)dlogits_dev % (dtype == OSSCAR_F32 ? 4 : 2)) bad = "osscar_logprobs_backward: dlogits is not aligned to its elements";
  if (!bad && dlogits_dev == logits_dev && ldd != ld && n > 1) bad = "osscar_logprobs_backward: in place, both leading dimensions are the same";
  if (bad) return refuse_call(OSSCAR_EINVAL, bad);
  hipStream_t s = reinterpret_cast<hipStream_t>(hip_stream);
  const size_t es = dtype == OSSCAR_F32 ? 4 : 2;
  for (int64_t r = 0; r < n; r += 65535) {      // (the grid's second dimension ends there)
    const int64_t rows = n - r < 65535 ? n - r : 65535;
    hipLaunchKernelGGL(logprobs_backward_kernel, dim3((unsigned)((vocab + CHUNK - 1) / CHUNK), (unsigned)rows), dim3(T), 0, s,
                       reinterpret_cast<const char*>(logits_dev) + r * ld * es, dtype == OSSCAR_F32, (int)vocab, ld, targets_dev + r, scale, lse_dev + 2 * r,
                       dlogp_dev ? dlogp_dev + r : nullptr, entropy_dev ? entropy_dev + r : nullptr, dentropy_dev ? dentropy_dev + r : nullptr, top,
                       top > 0 ? top_index_dev + r * top : nullptr, top > 0 ? dtop_dev + r * top : nullptr, reinterpret_cast<char*>(dlogits_dev) + r * ldd * es, ldd);
  }
  return launched("osscar_logprobs_backward");
}
