// The products of tile.h for float32 operands: C[m][n] = sum over segments and k of A[m][k] B[n][k] to the error of a float32 product, on the bf16 matrix cores.
//
// x = x1 + x2 + x3 with bf16 pieces of 8 bits each, and the six products of weight 2^-16 and more are summed in float32, the smallest first: 2.5 PFLOP/s / 6
// against the 157 TFLOP/s of the float32 instruction.  A stage (32 of the contraction) goes from memory to registers, is cut there and written to LDS as
// pieces, so that memory sees every operand as it is, at any alignment, and no pass over it is needed (pieces written out first: 22 bytes moved per weight
// instead of 4, which 128 rows through 7168 x 14336 paid with half their speed).  One set of stage buffers, the next two stages in registers, two workgroups
// per compute unit: while one cuts, the other multiplies.  4096 x 7168 x 14336: the pair of projections 8.9 ms (188 TFLOP/s; the library's float32 products
// 11.1), the backward pass 17.9 ms; operands whose rows begin at any 4 bytes (2048 x 1365 x 3001) 150 to 160 TFLOP/s.
#pragma once
#include "ops.h"
#include "tile.h"

namespace osscar {
namespace split {

using tile::OP_K;
using tile::OP_T;
using tile::Product;
using tile::Shape;
using tile::v4i;
using tile::v4s;

constexpr int KS = 32;      // contraction of a stage: one matrix-core operand

// Eight neighbouring values as pieces, each the nearest bf16 of what the ones before leave (of values below 1e-34 the last piece ends at bf16's smallest number,
// 9e-41).  What bf16 cannot hold as a finite number goes into the first
// piece alone, as it is (infinity, NaN) or cut off (the last float32 values).
__device__ __forceinline__ void cut(const float (&x)[8], v4i (&p)[3]) {
  float most = fabsf(x[0]);
#pragma unroll
  for (int e = 1; e < 8; e++) most = fmaxf(most, fabsf(x[e]));
  float sum = 0.f;      // NaN if one of them is
#pragma unroll
  for (int e = 0; e < 8; e++) sum += x[e] * 0.f;
  uint16_t w[3][8];
  if (most < 3.3e38f && sum == 0.f) {
#pragma unroll
    for (int e = 0; e < 8; e++) {
      w[0][e] = bf16_nearest(x[e]);
      const float r = x[e] - bf16_value(w[0][e]);
      w[1][e] = bf16_nearest(r);
      w[2][e] = bf16_nearest(r - bf16_value(w[1][e]));
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; e++) {
      const uint32_t u = __float_as_uint(x[e]);
      const bool finite = (u & 0x7F800000u) != 0x7F800000u;
      w[0][e] = finite ? (uint16_t)(u >> 16) : bf16_nearest(x[e]);
      const float r = finite ? x[e] - bf16_value(w[0][e]) : 0.f;
      w[1][e] = bf16_nearest(r);
      w[2][e] = bf16_nearest(r - bf16_value(w[1][e]));
    }
  }
#pragma unroll
  for (int t = 0; t < 3; t++) p[t] = __builtin_bit_cast(v4i, w[t]);
}

// One side, as tile::Side; the LDS rows of OP_K have four packets.
template <int MODE, int EXT, int PER, bool PERM>
struct Side {
  static constexpr int ROW = MODE == OP_K ? KS * 2 : EXT * 2, PK = ROW / 16, BYTES = EXT * KS * 2, NJ = EXT * KS / 8 / 256;
  static_assert(EXT * KS / 8 % 256 == 0, "");
  static __device__ __forceinline__ int swizzle(int row) {
    if (MODE == OP_K) {      // times two in the field of four elements, which differs over any four of the row groups that an access meets
      const int q = (row >> (PERM ? 3 : 2)) & 3;
      return ((q << 1) & 3) ^ ((q >> 1) * 3);
    }
    if (PERM) return PK == 8 ? (row & 2) << 1 : (row & 3) << 2;
    return (((row & 3) | (((row >> 3) & 1) << 2)) << 1) & (PK - 1);
  }
  const float* p[NJ];
  int r[NJ], c[NJ], at[NJ];      // row and first element along it of the thread's packets within the workgroup's operand, place in LDS
  __device__ __forceinline__ void open() {
#pragma unroll
    for (int j = 0; j < NJ; j++) {
      const int i = threadIdx.x + 256 * j;
      r[j] = i / PK;
      c[j] = i % PK * 8;
      at[j] = r[j] * ROW + ((i % PK) ^ swizzle(r[j])) * 16;
    }
  }
  __device__ __forceinline__ void place(const tile::Operand& o, int seg, int row0, int k) {
#pragma unroll
    for (int j = 0; j < NJ; j++)
      p[j] = reinterpret_cast<const float*>(o.p[seg] + (int64_t)((MODE == OP_K ? row0 : k) + r[j]) * o.ldb) + (MODE == OP_K ? k : row0) + c[j];
  }
  // the stage at k into registers, zeros outside the operand
  __device__ __forceinline__ void load(const tile::Operand& o, int row0, int k, float (&x)[NJ][8]) {
#pragma unroll
    for (int j = 0; j < NJ; j++) {
      const bool in = MODE == OP_K ? row0 + r[j] < o.rows : k + r[j] < o.rows;
      const int most = in ? o.cols - (MODE == OP_K ? k + c[j] : row0 + c[j]) : 0;
      if (most >= 8) {
        const f32x4 a = *reinterpret_cast<const f32x4_any*>(p[j]), b = *reinterpret_cast<const f32x4_any*>(p[j] + 4);
#pragma unroll
        for (int e = 0; e < 4; e++) { x[j][e] = a[e]; x[j][4 + e] = b[e]; }
      } else {
#pragma unroll
        for (int e = 0; e < 8; e++) {
          x[j][e] = 0.f;
          if (e < most) x[j][e] = p[j][e];
        }
      }
      p[j] = MODE == OP_K ? p[j] + KS : reinterpret_cast<const float*>(reinterpret_cast<const char*>(p[j]) + KS * o.ldb);
    }
  }
  __device__ __forceinline__ void store(const float (&x)[NJ][8], char (*lds)[BYTES]) const {
#pragma unroll
    for (int j = 0; j < NJ; j++) {
      v4i w[3];
      cut(x[j], w);
#pragma unroll
      for (int t = 0; t < 3; t++) *reinterpret_cast<v4i*>(lds[t] + at[j]) = w[t];
    }
  }
  int raddr[MODE == OP_K ? 1 : PER];
  __device__ __forceinline__ void open_read(int wpos, int lane) {
    const int i = lane & 15, g = lane >> 4, first = wpos * PER * 16;
    if (MODE == OP_K) {
      const int row = first + (PERM ? (i >> 2) * 8 + (i & 3) : i);
      raddr[0] = row * ROW + ((g ^ swizzle(row)) * 16);
    } else {
      const int k = g * 8 + (i >> 2), q = i & 3;
#pragma unroll
      for (int t = 0; t < PER; t++) {
        const int col = first + (PERM ? (t >> 1) * 32 + q * 8 + (t & 1) * 4 : t * 16 + q * 4);
        raddr[t] = k * ROW + (((col >> 3) ^ swizzle(k)) * 16) + ((col >> 2) & 1) * 8;
      }
    }
  }
  __device__ __forceinline__ v4i read(const char* lds, int t) const {
    if (MODE == OP_K) return *reinterpret_cast<const v4i*>(lds + raddr[0] + (PERM ? (t >> 1) * 32 + (t & 1) * 4 : t * 16) * ROW);
    typedef __attribute__((address_space(3))) v4s lds_v4s;
    const char* q = lds + raddr[MODE == OP_K ? 0 : t];
    const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)q), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)(q + 4 * ROW));
    return __builtin_bit_cast(v4i, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  }
};

template <int AM, int BMODE, class S, class Epi>
__device__ __forceinline__ void product_tile(const Product<S::NB>& q, const Epi& epi) {
  typedef Side<AM, S::BM, S::FM, false> SA;
  typedef Side<BMODE, S::BN, S::FN, true> SB;
  typedef float v4f __attribute__((ext_vector_type(4)));
  typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
  __shared__ __align__(1024) char la[3][SA::BYTES], lb[S::NB][3][SB::BYTES];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave / S::WN, wn = wave % S::WN;
  const int tiles_m = (q.M + S::BM - 1) / S::BM, tiles_n = (q.N + S::BN - 1) / S::BN;
  const tile::Share share = tile::share_of(blockIdx.x, tiles_m * tiles_n, q.whole, q.parts);
  int tm, tn;
  tile::tile_of(share.t, tiles_m, tiles_n, tm, tn);
  SA sa;
  SB sb[S::NB];
  sa.open();
  sa.open_read(wm, lane);
#pragma unroll
  for (int z = 0; z < S::NB; z++) { sb[z].open(); sb[z].open_read(wn, lane); }
  v4f acc[S::FM][S::NB][S::FN];
#pragma unroll
  for (int i = 0; i < S::FM; i++)
#pragma unroll
    for (int z = 0; z < S::NB; z++)
#pragma unroll
      for (int j = 0; j < S::FN; j++)
#pragma unroll
        for (int r = 0; r < 4; r++) acc[i][z][j][r] = 0;
  float xa[2][SA::NJ][8], xb[2][S::NB][SB::NJ][8];      // two stages under way
  const int per = (q.k + KS - 1) / KS, all = per * q.nseg, span = (all + share.parts - 1) / share.parts;      // stages of a segment, of all, of a part
  const int begin = min(all, share.part * span), total = min(all - begin, span);
  int seg = per > 0 ? begin / per : 0, k = per > 0 ? begin % per * KS : 0;
  bool anew = true;
  auto load = [&](int set) {      // the next stage
    if (anew) {
      sa.place(q.a, seg, tm * S::BM, k);
#pragma unroll
      for (int z = 0; z < S::NB; z++) sb[z].place(q.b[z], seg, tn * S::BN, k);
    }
    sa.load(q.a, tm * S::BM, k, xa[set]);
#pragma unroll
    for (int z = 0; z < S::NB; z++) sb[z].load(q.b[z], tn * S::BN, k, xb[set][z]);
    k += KS;
    anew = k >= q.k;
    if (anew) { k = 0; seg++; }
  };
  auto stage = [&](int set, bool more) {
    __syncthreads();      // the last stage's readers are done
    sa.store(xa[set], la);
#pragma unroll
    for (int z = 0; z < S::NB; z++) sb[z].store(xb[set][z], lb[z]);
    __syncthreads();
    if (more) load(set);
    // x3 y1 + x2 y2 + x1 y3 + x2 y1 + x1 y2 + x1 y1
    constexpr int PX[6] = {2, 1, 0, 1, 0, 0}, PY[6] = {0, 1, 2, 0, 1, 0};
    v4i fb[3][S::NB][S::FN];
#pragma unroll
    for (int t = 0; t < 3; t++)
#pragma unroll
      for (int z = 0; z < S::NB; z++)
#pragma unroll
        for (int j = 0; j < S::FN; j++) fb[t][z][j] = sb[z].read(lb[z][t], j);
#pragma unroll
    for (int i = 0; i < S::FM; i++) {
      v4i fa[3];
#pragma unroll
      for (int t = 0; t < 3; t++) fa[t] = sa.read(la[t], i);
      if constexpr (S::NB == 2) {
        // An activation's argument, whose sign decides RELU's slope: a stage's products are summed from zero and then added, one rounding to the size of the
        // whole sum in 32 of the contraction instead of six.  4096 x 2688 x 367: root mean square error 1.4e-7 of the values' instead of 5.6e-7 (the library's
        // float32 product: 9.3e-7), for 3 to 5% of the time.
#pragma unroll
        for (int z = 0; z < S::NB; z++)
#pragma unroll
          for (int j = 0; j < S::FN; j++) {
            v4f sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int t = 0; t < 6; t++)
              sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, fb[PY[t]][z][j]), __builtin_bit_cast(v8bf, fa[PX[t]]), sum, 0, 0, 0);
#pragma unroll
            for (int r = 0; r < 4; r++) acc[i][z][j][r] += sum[r];
          }
      } else {
#pragma unroll
        for (int t = 0; t < 6; t++)
#pragma unroll
          for (int j = 0; j < S::FN; j++)
            acc[i][0][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, fb[PY[t]][0][j]), __builtin_bit_cast(v8bf, fa[PX[t]]), acc[i][0][j], 0, 0, 0);
      }
    }
  };
  if (total > 0) load(0);
  if (total > 1) load(1);
  for (int st = 0; st < total; st += 2) {
    stage(0, st + 2 < total);
    if (st + 1 < total) stage(1, st + 3 < total);
  }
  const int i = lane & 15, g = lane >> 4;
  auto each = [&](auto put) {
#pragma unroll
    for (int f = 0; f < S::FM; f++) {
      const int m = tm * S::BM + (wm * S::FM + f) * 16 + i;
#pragma unroll
      for (int t = 0; t < S::FN; t += 2) {
        const int n = tn * S::BN + wn * S::FN * 16 + t * 16 + g * 8;
        float v[S::NB][8];
#pragma unroll
        for (int z = 0; z < S::NB; z++)
#pragma unroll
          for (int e = 0; e < 8; e++) v[z][e] = acc[f][z][t + e / 4][e % 4];
        if (m < q.M && n < q.N) put(m, n, v, q.N);
      }
    }
  };
  if (share.parts == 1) {
    epi.each(each);
  } else {
    float* sums = reinterpret_cast<float*>(q.sums) + (int64_t)share.slot * S::NB * S::BM * S::BN;
    each([&](int m, int n, const float (&v)[S::NB][8], int) {
#pragma unroll
      for (int z = 0; z < S::NB; z++) tile::put_sums(sums + (z * S::BM + m - tm * S::BM) * S::BN + n - tn * S::BN, v[z]);
    });
  }
}

}  // namespace split
}  // namespace osscar
