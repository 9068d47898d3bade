// Log probabilities of given tokens, entropy and largest alternatives from logits, and the gradient.
#include "ops.h"
#include <float.h>

// Products and sums are rounded each, but where fmaf says otherwise: the rounding of c2 m below has to be the same in every place.
#pragma clang fp contract(off)

using namespace osscar;

namespace {

constexpr float LOG2E = 1.44269504088896341f, LN2 = 0.69314718055994531f;

// Running state of a row's softmax: the largest logit m so far (raw, at least -FLT_MAX), S = sum 2^y and A = sum -y 2^y with
// y = c2 l - m2 <= 0, c2 = scale log2(e), m2 = c2 m rounded.  log sum exp = ln2 (m2 + log2 S) and entropy = ln2 (log2 S + A / S): sums of terms of one sign.
// The rounding of m2 cancels, since every y has the same one, as long as it is small: 2^y of the largest logit is two to the power of that rounding, at most 2^-5
// while |m2| < 2^20 (float32's 24 bits).  Beyond (rows masked with a large constant or with minus infinity, logits of such a size) y = c2 (l - m), rounded
// to its own size.  A row of minus infinities leaves S = 0; NaN and plus infinity make S NaN.
struct Stat { float m, S, A; };
__device__ __forceinline__ bool plain(float m, float c2) { return fabsf(m) * c2 < 0x1p20f; }
__device__ __forceinline__ float offset_of(float m, float c2) { return plain(m, c2) ? m * c2 : 0.f; }
// c2 m - m2: y = c2 (l - m) + this
__device__ __forceinline__ float rounding_of(float m, float c2) { return plain(m, c2) ? fmaf(m, c2, -(m * c2)) : 0.f; }
__device__ __forceinline__ void shift(Stat& s, float m, float c2) {      // the largest becomes m >= s.m: every y falls by d
  if (s.S != 0.f) {
    float d;
    if (plain(s.m, c2) && plain(m, c2)) d = s.m * c2 - m * c2;
    else d = (s.m - m) * c2 + rounding_of(m, c2) - rounding_of(s.m, c2);
    const float e = __builtin_amdgcn_exp2f(d);
    s.A = e * (s.A - fmaxf(d, -200.f) * s.S);
    s.S *= e;
  }
  s.m = m;
}
__device__ __forceinline__ void join(Stat& s, Stat o, float c2) {
  const float m = fmaxf(s.m, o.m);
  shift(s, m, c2);
  shift(o, m, c2);
  s.S += o.S;
  s.A += o.A;
}
__device__ __forceinline__ float entropy_of(const Stat& s) { return s.S == 0.f ? 0.f : logf(s.S) + LN2 * (s.A / s.S); }
// log sum exp(scale (l - m))
__device__ __forceinline__ float log_sum_of(const Stat& s, float c2) { return s.S == 0.f ? -INFINITY : logf(s.S) - LN2 * rounding_of(s.m, c2); }
// scale (l - m), where the difference may be no float though the result is one
__device__ __forceinline__ float scaled(float l, float m, float scale) {
  const float d = l - m;
  return fabsf(d) < INFINITY ? scale * d : scale * l - scale * m;
}
// (not by way of c2: log2(e) times the lowest value, which masks are made of, is no float)
__device__ __forceinline__ float logp_of(const Stat& s, float l, float scale, float c2) {
  return s.S == 0.f ? -INFINITY : scaled(l, s.m, scale) - log_sum_of(s, c2);
}

// Order of alternatives: larger value first, then lower index; NaN above all, the two zeros equal.
__device__ __forceinline__ uint64_t rank_of(float l, uint32_t v) {
  uint32_t b = __float_as_uint(l + 0.f);
  if (l != l) b = 0x7FC00000u;
  b ^= (b & 0x80000000u) ? 0xFFFFFFFFu : 0x80000000u;
  return (uint64_t)b << 32 | (0xFFFFFFFFu - v);
}
__device__ __forceinline__ uint32_t index_of(uint64_t r) { return 0xFFFFFFFFu - (uint32_t)r; }
__device__ __forceinline__ float logit_of(uint64_t r) {
  const uint32_t b = (uint32_t)(r >> 32);
  return __uint_as_float(b & 0x80000000u ? b ^ 0x80000000u : ~b);
}

__device__ __forceinline__ float logit(const void* p, int f32, int64_t at) {
  return f32 ? reinterpret_cast<const float*>(p)[at] : bf16_value(reinterpret_cast<const uint16_t*>(p)[at]);
}

// Eight neighbouring logits as they are in memory
template <bool F32> struct Packet;
template <> struct Packet<false> {
  typedef u16x8 type;
  static __device__ __forceinline__ type at(const void* p, int64_t i) { return *reinterpret_cast<const u16x8_any*>(reinterpret_cast<const uint16_t*>(p) + i); }
  static __device__ __forceinline__ type some(const void* p, int64_t i, int most) {      // minus infinity after `most` of them
    type w;
#pragma unroll
    for (int e = 0; e < 8; e++) w[e] = e < most ? reinterpret_cast<const uint16_t*>(p)[i + e] : (uint16_t)0xFF80;
    return w;
  }
  static __device__ __forceinline__ void values(const type& w, float (&l)[8]) {
#pragma unroll
    for (int e = 0; e < 8; e++) l[e] = bf16_value(w[e]);
  }
};
template <> struct Packet<true> {
  struct type { f32x4 a, b; };
  static __device__ __forceinline__ type at(const void* p, int64_t i) {
    const float* q = reinterpret_cast<const float*>(p) + i;
    return type{*reinterpret_cast<const f32x4_any*>(q), *reinterpret_cast<const f32x4_any*>(q + 4)};
  }
  static __device__ __forceinline__ type some(const void* p, int64_t i, int most) {
    const float* q = reinterpret_cast<const float*>(p) + i;
    type w;
#pragma unroll
    for (int e = 0; e < 4; e++) { w.a[e] = e < most ? q[e] : -INFINITY; w.b[e] = e + 4 < most ? q[e + 4] : -INFINITY; }
    return w;
  }
  static __device__ __forceinline__ void values(const type& w, float (&l)[8]) {
#pragma unroll
    for (int e = 0; e < 4; e++) { l[e] = w.a[e]; l[e + 4] = w.b[e]; }
  }
};

constexpr int T = 256, EACH = 4;             // threads; packets of eight logits that a thread has under way
constexpr int BATCH = T * 8 * EACH;          // logits of a step of a workgroup
constexpr int CANDS = 1024;                  // packets that a workgroup can list
static_assert(CANDS >= T * EACH && CANDS >= 8 * OSSCAR_TOP_MAX, "a whole first step fits, and so do the logits of the chosen packets");
constexpr int JOIN = 1024;                   // alternatives of a row's parts together, at most

struct Row {      // what a row's results go to
  const int64_t* targets; float scale; int top; float *logp, *entropy, *lse; int64_t* top_index; float* top_logp;
};
struct Given { int64_t t; float l; };      // a row's target and its logit, fetched before the row so that nothing waits for them at its end
__device__ __forceinline__ Given given(const Row& o, const void* logits, int f32, int vocab, int64_t base, int64_t row) {
  const int64_t t = o.targets[row];
  return Given{t, t >= 0 && t < vocab ? logit(logits, f32, base + t) : NAN};
}
__device__ __forceinline__ void put_row(const Row& o, int64_t row, const Stat& s, Given g, float c2) {
  o.logp[row] = g.t < 0 ? 0.f : (g.l == g.l ? logp_of(s, g.l, o.scale, c2) : NAN);
  if (o.entropy) o.entropy[row] = entropy_of(s);
  if (o.lse) { o.lse[2 * row] = s.m; o.lse[2 * row + 1] = log_sum_of(s, c2); }
}
__device__ __forceinline__ uint64_t max_of_block(uint64_t best, uint64_t* sh) {      // sh: T / 64 words
  for (int o = 32; o > 0; o >>= 1) { const uint64_t x = __shfl_xor((unsigned long long)best, o, 64); best = x > best ? x : best; }
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = best;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < T / 64; w++) best = sh[w] > best ? sh[w] : best;
  return best;
}
// The k largest of n ranks in LDS: each thread counts how many are above its own, put(place, rank).
template <class F>
__device__ __forceinline__ void choose(const uint64_t* ranks, int n, int k, F put) {
  for (int i = threadIdx.x; i < n; i += T) {
    const uint64_t r = ranks[i];
    int above = 0;
#pragma unroll 8
    for (int j = 0; j < n; j++) above += ranks[j] > r;
    if (above < k) put(above, r);
  }
}

// A part of a row per workgroup (blockIdx.y of `parts`), read once: softmax statistics and the candidates for the alternatives.
// The k largest logits lie in the k packets whose largest logit ranks highest (of equal ones the first packet).  After the first step, which holds the lowest
// indices, the k-th largest of the threads' (groups of threads') maxima is a lower bound of the k-th packet's, and k packets of that step are not below it.
// They go into a list with their maxima, and so does every later packet above it (an equal one loses by its index): a few times k of random logits, whatever
// the row's length; a step where no thread has one costs a comparison per 32 logits.  At the end the k best packets are chosen by counting, read again, and the
// k best logits in them chosen likewise.  Where the list is too short (ever larger logits; a first step with a mask's value in all but fewer than k groups), or
// with NaN and infinity, the part is read k times more.
// Bound by reading the logits (4096 x 50304 bf16, five alternatives: 89 us, 4.6 TB/s; float32 6.0 TB/s); per logit about 10 slots of the vector unit, four of
// them the exponential.
template <bool F32>
__global__ __launch_bounds__(T) void logprobs_kernel(const void* __restrict__ logits, int vocab, int64_t ld, int span, Row out, Stat* part_stat, uint64_t* part_rank) {
  __shared__ Stat st[T / 64];
  __shared__ float maxima[T];
  __shared__ float bound_sh;
  __shared__ int count, count2;
  __shared__ uint64_t cand[CANDS], chosen[OSSCAR_TOP_MAX], sh[T / 64];
  const int64_t row = blockIdx.x, base = row * ld;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int c0 = blockIdx.y * span, c1 = min(vocab, c0 + span), k = min(out.top, c1 - c0);
  const float c2 = out.scale * LOG2E;
  Given g{-1, 0.f};
  if (tid == 0 && !part_stat) g = given(out, logits, F32, vocab, base, row);
  Stat s{-FLT_MAX, 0.f, 0.f};
  float m2 = offset_of(s.m, c2), bound = INFINITY;
  if (tid == 0) count = count2 = 0;
  auto from_row = [&](int v0, int v1, auto put) {      // the k largest of [v0, v1) one by one, by thread 0
    uint64_t last = ~0ull;
    for (int j = 0; j < k; j++) {
      uint64_t best = 0;
      for (int v = v0 + tid; v < v1; v += T) {
        const uint64_t r = rank_of(logit(logits, F32, base + v), v);
        if (r < last && r > best) best = r;
      }
      last = max_of_block(best, sh);
      if (tid == 0) put(j, last);
    }
  };
  typedef typename Packet<F32>::type P;
  auto fetch = [&](int b, P (&p)[EACH]) {
    if (b + BATCH <= c1) {
#pragma unroll
      for (int u = 0; u < EACH; u++) p[u] = Packet<F32>::at(logits, base + b + (u * T + tid) * 8);
    } else {
#pragma unroll
      for (int u = 0; u < EACH; u++) {
        const int v0 = b + (u * T + tid) * 8;
        if (v0 + 8 <= c1) p[u] = Packet<F32>::at(logits, base + v0);
        else p[u] = Packet<F32>::some(logits, base + v0, c1 - v0);
      }
    }
  };
  for (int b = c0; b < c1; b += BATCH) {
    P p[EACH];
    float l[EACH][8];
    fetch(b, p);
#pragma unroll
    for (int u = 0; u < EACH; u++) Packet<F32>::values(p[u], l[u]);
    float most = -INFINITY, packet[EACH];
#pragma unroll
    for (int u = 0; u < EACH; u++) {
      packet[u] = l[u][0];
#pragma unroll
      for (int e = 1; e < 8; e++) packet[u] = fmaxf(packet[u], l[u][e]);
      most = fmaxf(most, packet[u]);
    }
    if (most > s.m) { shift(s, most, c2); m2 = offset_of(most, c2); }
    if (plain(s.m, c2)) {
      float S = 0.f, A = 0.f;
#pragma unroll
      for (int u = 0; u < EACH; u++)
#pragma unroll
        for (int e = 0; e < 8; e++) {
          const float y = fmaf(l[u][e], c2, -m2), x = __builtin_amdgcn_exp2f(y);
          S += x;
          A = fmaf(fmaxf(y, -200.f), x, A);      // (2^-200 is 0: y = -inf adds nothing)
        }
      s.S += S;
      s.A -= A;
    } else {
      for (int u = 0; u < EACH; u++)
        for (int e = 0; e < 8; e++) {
          const float y = (l[u][e] - s.m) * c2, x = __builtin_amdgcn_exp2f(y);
          s.S += x;
          s.A -= fmaxf(y, -200.f) * x;
        }
    }
    if (k > 0) {
      if (b == c0) {
        // maxima of 16, 4 or 1 threads: at least twice as many as alternatives
        const int per = k <= 8 ? 16 : k <= 32 ? 4 : 1, groups = T / per;
        float g = most;
        for (int o = per / 2; o > 0; o >>= 1) g = fmaxf(g, __shfl_xor(g, o, 64));
        if (tid % per == 0) maxima[tid / per] = g;
        __syncthreads();
        if (tid < groups) {
          const float mine = maxima[tid];
          int above = 0;
          for (int j = 0; j < groups; j++) above += maxima[j] > mine || (maxima[j] == mine && j < tid);
          if (above == k - 1) bound_sh = mine;
        }
        __syncthreads();
        bound = bound_sh;
      }
      if (most >= bound) {
#pragma unroll
        for (int u = 0; u < EACH; u++) {
          const int v0 = b + (u * T + tid) * 8;
          if (packet[u] >= bound && v0 < c1) {
            const int at = atomicAdd(&count, 1);
            if (at < CANDS) cand[at] = rank_of(packet[u], v0);
          }
        }
      }
      if (b == c0) bound = nextafterf(bound, INFINITY);      // from here on above it
    }
  }
  for (int o = 32; o > 0; o >>= 1) join(s, Stat{__shfl_xor(s.m, o, 64), __shfl_xor(s.S, o, 64), __shfl_xor(s.A, o, 64)}, c2);
  if (lane == 0) st[wave] = s;
  __syncthreads();
  s = st[0];
#pragma unroll
  for (int w = 1; w < T / 64; w++) join(s, st[w], c2);
  if (tid == 0) {
    if (part_stat) part_stat[row * gridDim.y + blockIdx.y] = s;
    else put_row(out, row, s, g, c2);
  }
  if (out.top == 0) return;
  auto put = [&](int j, uint64_t r) {
    if (part_rank) {
      part_rank[(row * gridDim.y + blockIdx.y) * out.top + j] = r;
    } else {
      out.top_index[row * out.top + j] = index_of(r);
      out.top_logp[row * out.top + j] = logp_of(s, logit_of(r), out.scale, c2);
    }
  };
  if (part_rank && tid >= k && tid < out.top) put(tid, 0);      // a part shorter than that (ranks of logits are above 0)
  const int n = count;
  if (n > CANDS || s.S != s.S) {
    from_row(c0, c1, put);
    return;
  }
  const int packets = min(n, k);
  choose(cand, n, packets, [&](int j, uint64_t r) { chosen[j] = r; });
  __syncthreads();
  if (packets > 0) {      // (no part is without a packet, but for those past the row's end)
    const float least = packets < k ? -INFINITY : logit_of(chosen[k - 1]);
    for (int i = tid; i < packets * 8; i += T) {
      const int v = (int)index_of(chosen[i >> 3]) + (i & 7);
      if (v >= c1) continue;
      const float x = logit(logits, F32, base + v);
      if (x >= least) cand[atomicAdd(&count2, 1)] = rank_of(x, v);
    }
  }
  __syncthreads();
  choose(cand, count2, k, put);
}
// The parts of a row put together, a row per workgroup: 4 x 131072 float32 13 us for both launches with eight alternatives, 22 us with 64, 8 us without.
__global__ __launch_bounds__(T) void logprobs_join_kernel(const void* __restrict__ logits, int f32, int vocab, int64_t ld, int parts, Row out,
                                                          const Stat* __restrict__ part_stat, const uint64_t* __restrict__ part_rank) {
  __shared__ uint64_t ranks[JOIN], best[JOIN];
  __shared__ int count;
  const int64_t row = blockIdx.x, base = row * ld;
  const float c2 = out.scale * LOG2E;
  const int lane = threadIdx.x & 63;
  Given g{-1, 0.f};
  if (threadIdx.x == 0) g = given(out, logits, f32, vocab, base, row);
  Stat s = lane < parts ? part_stat[row * parts + lane] : Stat{-FLT_MAX, 0.f, 0.f};      // (at most 64 parts; every wave for itself)
  for (int o = 32; o > 0; o >>= 1) join(s, Stat{__shfl_xor(s.m, o, 64), __shfl_xor(s.S, o, 64), __shfl_xor(s.A, o, 64)}, c2);
  if (threadIdx.x == 0) put_row(out, row, s, g, c2);
  if (out.top == 0) return;
  // A part's alternatives come in order.  With c parts whose m-th is not below some rank, c m >= top are not, and what is below it is out: about half the parts
  // give a rank that few others reach.
  const int n = parts * out.top, m = min(out.top, (2 * out.top + parts - 1) / parts), c = (out.top + m - 1) / m;
  for (int i = threadIdx.x; i < n; i += T) ranks[i] = part_rank[row * n + i];
  if (threadIdx.x == 0) count = 0;
  __syncthreads();
  const uint64_t mine = lane < parts ? ranks[lane * out.top + m - 1] : 0;
  int above = 0;
#pragma unroll 8
  for (int j = 0; j < parts; j++) above += ranks[j * out.top + m - 1] > mine;
  const uint64_t at = __ballot(above == c - 1 && lane < parts);      // (no lane: short parts, whose missing ones are 0)
  const uint64_t bound = at ? (uint64_t)__shfl((unsigned long long)mine, __ffsll((unsigned long long)at) - 1, 64) : 0;
  for (int i = threadIdx.x; i < n; i += T)
    if (ranks[i] > 0 && ranks[i] >= bound) best[atomicAdd(&count, 1)] = ranks[i];
  __syncthreads();
  choose(best, count, out.top, [&](int j, uint64_t r) {
    out.top_index[row * out.top + j] = index_of(r);
    out.top_logp[row * out.top + j] = logp_of(s, logit_of(r), out.scale, c2);
  });
}
// Parts of a row: as many as give two workgroups per compute unit, each of at least a packet per thread, whose alternatives fit the join.
int parts_of(int64_t n, int64_t vocab, int32_t top) {
  int64_t parts = n > 0 ? 512 / n : 1;
  const int64_t most = (vocab + T * 8 - 1) / (T * 8);
  if (parts > most) parts = most;
  if (parts > 64) parts = 64;
  if (top > 0 && parts > JOIN / top) parts = JOIN / top;
  return parts < 1 ? 1 : (int)parts;
}

// Gradient.  A workgroup takes CHUNK columns of a row; the few columns that have a term of their own (target, alternatives) are computed by a
// thread each from logits read before the others are written.  Bound by reading and writing: 8192 x 32000 bf16 187 us, 5.6 TB/s.
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
  const bool empty = lnS == -INFINITY, large = m > 1e30f;      // (only of such a maximum may a difference of logits be no float)
  auto grad = [&](float l, float own) {
    const float lp = (large ? scaled(l, m, scale) : scale * (l - m)) - lnS, p = __expf(lp);
    const float x = -p * (w + (p == 0.f ? 0.f : dh * (lp + H)));      // (w of no number makes the whole row so)
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
  if (!(scale > 0.f && scale * LOG2E < INFINITY)) return "osscar_logprobs: scale must be positive and below 2.3e38";
  if (top < 0 || top > OSSCAR_TOP_MAX || top > vocab) return "osscar_logprobs: top is at most OSSCAR_TOP_MAX and at most vocab";
  if (n > 0 && (!logits || !targets || ld < vocab)) return "osscar_logprobs: NULL pointer or leading dimension below the row length";
  if ((uintptr_t)logits % (dtype == OSSCAR_F32 ? 4 : 2)) return "osscar_logprobs: logits are not aligned to their elements";
  return nullptr;
}

}  // namespace

extern "C" size_t osscar_logprobs_workspace_bytes(int64_t n, int64_t vocab, int32_t top) {
  if (!a_size(n, 0) || !a_size(vocab, 1) || top < 0 || top > OSSCAR_TOP_MAX || top > vocab) return 0;
  const int parts = parts_of(n, vocab, top);
  Carve c(nullptr);
  if (parts > 1) {
    c.take((size_t)n * parts * sizeof(Stat));
    c.take((size_t)n * parts * top * 8);
  }
  return c.used + 256;
}

extern "C" osscar_status osscar_logprobs(const void* logits_dev, int64_t n, int64_t vocab, int64_t ld, int32_t dtype, const int64_t* targets_dev, float scale,
                                         int32_t top, float* logp_dev, float* entropy_dev, float* lse_dev, int64_t* top_index_dev, float* top_logp_dev,
                                         void* workspace_dev, size_t workspace_bytes, void* hip_stream) {
  const char* bad = bad_logits(logits_dev, n, vocab, ld, dtype, targets_dev, scale, top);
  if (!bad && n > 0 && (!logp_dev || (top > 0 && (!top_index_dev || !top_logp_dev)))) bad = "osscar_logprobs: NULL pointer";
  if (!bad && ((uintptr_t)workspace_dev & 255)) bad = "osscar_logprobs: the workspace must begin at a 256-byte boundary";
  if (bad) return refuse_call(OSSCAR_EINVAL, bad);
  if (n == 0) return OSSCAR_OK;
  hipStream_t s = reinterpret_cast<hipStream_t>(hip_stream);
  const int f32 = dtype == OSSCAR_F32, parts = parts_of(n, vocab, top);
  const int span = (int)((vocab + parts - 1) / parts + 7) / 8 * 8;
  const Row out{targets_dev, scale, top, logp_dev, entropy_dev, lse_dev, top_index_dev, top_logp_dev};
  Stat* stat = nullptr;
  uint64_t* rank = nullptr;
  if (parts > 1) {
    Carve c(workspace_dev);
    stat = reinterpret_cast<Stat*>(c.take((size_t)n * parts * sizeof(Stat)));
    rank = reinterpret_cast<uint64_t*>(c.take((size_t)n * parts * top * 8));
    if (!workspace_dev || c.used > workspace_bytes) return refuse_call(OSSCAR_ENOMEM, "osscar_logprobs: workspace too small");
  }
  constexpr int64_t LAUNCH = 1 << 23;      // rows: a launch has fewer than 2^32 threads along a dimension (many rows are in one part)
  const size_t es = f32 ? 4 : 2;
  for (int64_t r = 0; r < n; r += LAUNCH) {
    const dim3 grid((unsigned)(n - r < LAUNCH ? n - r : LAUNCH), (unsigned)parts);
    const void* from = reinterpret_cast<const char*>(logits_dev) + r * ld * es;
    const Row to{targets_dev + r, scale, top, logp_dev + r, entropy_dev ? entropy_dev + r : nullptr, lse_dev ? lse_dev + 2 * r : nullptr,
                 top > 0 ? top_index_dev + r * top : nullptr, top > 0 ? top_logp_dev + r * top : nullptr};
    if (f32) hipLaunchKernelGGL(logprobs_kernel<true>, grid, dim3(T), 0, s, from, (int)vocab, ld, span, to, stat, rank);
    else hipLaunchKernelGGL(logprobs_kernel<false>, grid, dim3(T), 0, s, from, (int)vocab, ld, span, to, stat, rank);
  }
  if (parts > 1) hipLaunchKernelGGL(logprobs_join_kernel, dim3((unsigned)n), dim3(T), 0, s, logits_dev, f32, (int)vocab, ld, parts, out, stat, rank);
  return launched();
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
  if (n == 0) return OSSCAR_OK;
  hipStream_t s = reinterpret_cast<hipStream_t>(hip_stream);
  const size_t es = dtype == OSSCAR_F32 ? 4 : 2;
  for (int64_t r = 0; r < n; r += 65535) {      // (the grid's second dimension ends there)
    const int64_t rows = n - r < 65535 ? n - r : 65535;
    hipLaunchKernelGGL(logprobs_backward_kernel, dim3((unsigned)((vocab + CHUNK - 1) / CHUNK), (unsigned)rows), dim3(T), 0, s,
                       reinterpret_cast<const char*>(logits_dev) + r * ld * es, dtype == OSSCAR_F32, (int)vocab, ld, targets_dev + r, scale, lse_dev + 2 * r,
                       dlogp_dev ? dlogp_dev + r : nullptr, entropy_dev ? entropy_dev + r : nullptr, dentropy_dev ? dentropy_dev + r : nullptr, top,
                       top > 0 ? top_index_dev + r * top : nullptr, top > 0 ? dtop_dev + r * top : nullptr, reinterpret_cast<char*>(dlogits_dev) + r * ldd * es, ldd);
  }
  return launched();
}
