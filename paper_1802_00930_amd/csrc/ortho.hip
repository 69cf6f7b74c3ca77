// Orthogonalised updates (see dfp.h): X = U / (|U| + eps), then steps of
//   A = X X^T, B = b A + c A A, X = a X + B X
// with the smaller side first (X^T X and X B where rows > cols).
//
// The products read f16 operands in the layout of mma_tile.h: `gram` is X (or X^T
// where R > C) with its longer side contiguous, `step` the other of the two; both
// are written by the kernel that makes X.  X is held as the sum of two f16 numbers
// (2^-24 of a value).  BF16 results: the operands are the high one alone, the low one
// lies beside them, [R][C]; otherwise the operands have both.  All sides are padded
// to 64 with zeros, which every step keeps zero.
//
// A and B are symmetric: only tiles on and above the diagonal are computed and each
// is stored twice.  a X joins in FP32 (with a in B's operand, where it would be off by
// 2^-23, the result is three times as far off for matrices of strong directions above
// weak ones).  In an operand of one f16 number B's diagonal, the largest entries of its
// rows, would be off by most: it stays out and joins too, X = (a + B_ii) X + B' X.
//
// Weight steps of matrices that are much longer one way take several iterations on
// the small square before X is touched: with P = a I + B, the next A is P A P (all are
// polynomials of A: they commute, and their products are symmetric), and
// X = P_2 P_1 X = q X + Q X with q = a_2 a_1, Q = a_2 B_1 + a_1 B_2 + B_2 B_1.  That replaces a
// Gram product and a step by three products of the small side.  An error of A grows by
// the square of P's norm an iteration, m = a^2 where a is the largest that a + b s + c s^2
// gets on [0, 1], and enters the next polynomial by its slope, |b| + 2 |c| at most.  So A is
// computed from X again once m m' is above 150 (two iterations of a = 3.44) or, times the next
// slope, above 1600 (1244 there): 2^-22 of A become 4e-4 of the update at worst, and measured
// up to 4e-5 with those coefficients, where single iterations and FP32 products may end at
// 1e-6, of an update that enters FP32 weights times lr.
//
// Units: X in 2^-12, A in 2^-10, which hold singular values up to 4 twice over; B and Q in
// one that holds what such values, before and after the step, can make of them (unit_b, run).
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "dfp_internal.h"
#include "dfp_types.h"
#include "mma_tile.h"
#include "ortho.h"

#pragma clang fp contract(off)

namespace dfp {

namespace {

constexpr int kBlock = 256;
constexpr int kUnitX = 12, kUnitA = 10;
constexpr int kNormParts = 1024;  // most partial sums of a matrix

struct Plan {
  bool tall;             // rows > cols
  int64_t R, C, Rp, Cp;  // the matrix, padded
  int64_t r, rp;         // the smaller side, padded
  int64_t e;             // bytes of an operand element
  int64_t xlo, gram, step0, step1, aa, bb, pa, qq0, qq1, diag, norm, slices, bytes;  // offsets, total
  OrthoPlan mm;
};

Plan make_plan(const dfp_ortho_desc& d, bool split) {
  Plan p;
  p.R = d.rows;
  p.C = d.cols;
  p.tall = d.rows > d.cols;
  p.Rp = (p.R + 63) / 64 * 64;
  p.Cp = (p.C + 63) / 64 * 64;
  p.r = p.tall ? p.C : p.R;
  p.rp = p.tall ? p.Cp : p.Rp;
  p.e = split ? 4 : 2;
  int64_t at = 0;
  auto take = [&](int64_t bytes) {
    const int64_t o = at;
    at += (bytes + 255) / 256 * 256;
    return o;
  };
  const int64_t n = p.Rp * p.Cp * d.batch, s = p.rp * p.rp * d.batch;
  p.mm = plan_ortho(d.batch, p.R, p.C, split);
  p.xlo = take(split ? 0 : n * 2);
  p.gram = take(n * p.e);
  p.step0 = take(n * p.e);
  p.step1 = take(n * p.e);
  p.aa = take(s * p.e);
  p.bb = take(s * p.e);
  p.pa = take(p.mm.grouped ? s * p.e : 0);
  p.qq0 = take(p.mm.grouped ? s * p.e : 0);
  p.qq1 = take(p.mm.grouped ? s * p.e : 0);
  p.diag = take(split ? 0 : p.rp * d.batch * 4);
  p.norm = take((int64_t)kNormParts * d.batch * 8);
  p.slices = take(p.mm.gram.bytes);
  p.bytes = at;
  return p;
}

// ---------------------------------------------------------------- operands
// Byte offset of element k of a row.
template <Prod P>
__device__ __forceinline__ int64_t op_off(int64_t k) {
  return P == Prod::F16X2 ? (k >> 5) * 128 + (k & 31) * 2 : k * 2;
}
__device__ __forceinline__ uint16_t h_bits(_Float16 h) { return __builtin_bit_cast(uint16_t, h); }
__device__ __forceinline__ float h_val(uint32_t b) { return (float)__builtin_bit_cast(_Float16, (uint16_t)b); }

// v (in units already) to elements of the row at p: four k .. k + 3, k a multiple of 4,
// or eight.
template <Prod P>
__device__ __forceinline__ void put4(uint8_t* p, int64_t k, const float (&v)[4]) {
  uint32_t hi[4], lo[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const _Float16 h = (_Float16)v[i];
    hi[i] = h_bits(h);
    lo[i] = h_bits((_Float16)(v[i] - (float)h));
  }
  uint2* d = (uint2*)(p + op_off<P>(k));
  d[0] = make_uint2(hi[0] | hi[1] << 16, hi[2] | hi[3] << 16);
  if (P == Prod::F16X2) d[8] = make_uint2(lo[0] | lo[1] << 16, lo[2] | lo[3] << 16);
}
__device__ __forceinline__ uint4 pack8(const float (&v)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = h_bits((_Float16)v[2 * i]) | (uint32_t)h_bits((_Float16)v[2 * i + 1]) << 16;
  return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ uint4 pack8_low(const float (&v)[8]) {
  float l[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) l[i] = v[i] - (float)(_Float16)v[i];
  return pack8(l);
}
template <Prod P>
__device__ __forceinline__ void put8(uint8_t* p, int64_t k, const float (&v)[8]) {
  uint4* d = (uint4*)(p + op_off<P>(k));
  d[0] = pack8(v);
  if (P == Prod::F16X2) d[4] = pack8_low(v);
}
__device__ __forceinline__ void unpack8(const uint4& h, const uint4& l, float (&v)[8]) {
  const uint32_t hw[4] = {h.x, h.y, h.z, h.w}, lw[4] = {l.x, l.y, l.z, l.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = h_val(hw[i]) + h_val(lw[i]);
    v[2 * i + 1] = h_val(hw[i] >> 16) + h_val(lw[i] >> 16);
  }
}

// -------------------------------------------------------------------- norm
// u = x (v null), or the momentum step on v in place and u from it.
template <int T>
struct Source {
  const typename Elem<T>::type* x;
  float* v;
  float mu;
  bool nesterov;
};
// (its elements fetched before, g and the new v)
template <int T, bool MUON>
__device__ __forceinline__ void direction(const Source<T>& s, const Raw<T, 4>& g, const Raw<DFP_F32, 4>& vnew,
                                          float (&u)[4]) {
  up_n<T, 4>(g, u);
  if (MUON) {
    float v[4];
    up_n<DFP_F32, 4>(vnew, v);
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = s.nesterov ? fmaf(s.mu, v[i], u[i]) : v[i];
  }
}

// Momentum update and partial sums of u^2 (in 64 bits), gridDim.x a matrix.  Bound by
// memory: 2048 x 8192 FP32 with momentum 39 us (5.2 TB/s).
template <int T, bool MUON>
__global__ __launch_bounds__(kBlock) void k_norm(Source<T> s, int64_t n, double* __restrict__ part) {
  __shared__ double red[kBlock / 64];
  const int64_t base = (int64_t)blockIdx.y * n, stride = (int64_t)gridDim.x * kBlock * 4;
  double sum = 0.;
  constexpr int U = 4;  // quads in flight
  for (int64_t i = ((int64_t)blockIdx.x * kBlock + threadIdx.x) * 4; i < n; i += stride * U) {
    Raw<T, 4> raw[U];
    Raw<DFP_F32, 4> old[MUON ? U : 1];
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const int64_t at = i + k * stride;
      fetch_n<T, 4>(s.x + base + at, n - at, raw[k]);
      if (MUON) fetch_n<DFP_F32, 4>(s.v + base + at, n - at, old[k]);
    }
    float g[U][4], v[U][4];
#pragma unroll
    for (int k = 0; k < U; ++k) {
      up_n<T, 4>(raw[k], g[k]);
      if (MUON) up_n<DFP_F32, 4>(old[k], v[k]);
    }
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const int64_t at = i + k * stride;
      if (MUON) {
        float u[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          v[k][j] = fmaf(s.mu, v[k][j], g[k][j]);
          u[j] = s.nesterov ? fmaf(s.mu, v[k][j], g[k][j]) : v[k][j];
          sum += (double)u[j] * (double)u[j];
        }
        store_n<DFP_F32, 4>(s.v + base + at, n - at, v[k]);
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) sum += (double)g[k][j] * (double)g[k][j];
      }
    }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x == 0)
    part[(int64_t)blockIdx.y * gridDim.x + blockIdx.x] = (red[0] + red[1]) + (red[2] + red[3]);
}

// X = u / (|u| + eps): both operands (and the low parts), 64 x 64 tiles of the padded matrix.
// Bound by memory: 2048 x 8192 FP32 with momentum 56 us (4.8 TB/s).
template <int T, bool MUON, Prod P>
__global__ __launch_bounds__(kBlock) void k_pack(Source<T> s, int64_t R, int64_t C, int64_t Rp, int64_t Cp,
                                                 const double* __restrict__ part, int32_t parts, float eps,
                                                 uint16_t* __restrict__ xlo, uint8_t* __restrict__ rowop,
                                                 uint8_t* __restrict__ colop) {
  __shared__ float tile[64][65];
  __shared__ double red[kBlock / 64];
  const int64_t b = blockIdx.y;
  const int64_t ct = Cp / 64, r0 = blockIdx.x / ct * 64, c0 = blockIdx.x % ct * 64;
  const int cc = (threadIdx.x & 15) * 4;
  double sums[kNormParts / kBlock];
#pragma unroll
  for (int i = 0; i < kNormParts / kBlock; ++i) {
    const int32_t at = threadIdx.x + i * kBlock;
    sums[i] = at < parts ? part[b * parts + at] : 0.;
  }
  Raw<T, 4> raw[4];
  Raw<DFP_F32, 4> vnew[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t r = r0 + (threadIdx.x >> 4) + i * 16, c = c0 + cc, at = (b * R + r) * C + c;
    fetch_n<T, 4>(s.x + at, r < R ? C - c : 0, raw[i]);
    if (MUON) fetch_n<DFP_F32, 4>(s.v + at, r < R ? C - c : 0, vnew[i]);
  }
  float u[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i) direction<T, MUON>(s, raw[i], vnew[i], u[i]);
  double sum = (sums[0] + sums[1]) + (sums[2] + sums[3]);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = sum;
  __syncthreads();
  const double nrm = sqrt((red[0] + red[1]) + (red[2] + red[3]));
  const double inv = isfinite(nrm) ? 1. / (nrm + (double)eps) : (double)__uint_as_float(0x7fc00000u);
  constexpr int64_t e = P == Prod::F16X2 ? 4 : 2;
  const int64_t pbytes = Rp * Cp * e;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int rr = (threadIdx.x >> 4) + i * 16;
    const int64_t r = r0 + rr, c = c0 + cc;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      u[i][j] = r < R && c + j < C ? (float)((double)u[i][j] * inv) * (float)(1 << kUnitX) : 0.f;
      tile[rr][cc + j] = u[i][j];
    }
    put4<P>(rowop + b * pbytes + r * Cp * e, c, u[i]);
    if (P == Prod::F16) {
      uint16_t lo[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) lo[j] = h_bits((_Float16)(u[i][j] - (float)(_Float16)u[i][j]));
      *(uint2*)(xlo + (b * Rp + r) * Cp + c) = make_uint2(lo[0] | (uint32_t)lo[1] << 16, lo[2] | (uint32_t)lo[3] << 16);
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int rr = (threadIdx.x >> 4) + i * 16;
    const float v[4] = {tile[cc][rr], tile[cc + 1][rr], tile[cc + 2][rr], tile[cc + 3][rr]};
    put4<P>(colop + b * pbytes + (c0 + rr) * Rp * e, r0 + cc, v);
  }
}

// ---------------------------------------------------------------- products
struct MmArgs {
  const uint8_t *a, *b;    // operands, of one batch element
  int64_t lda, ldb;        // bytes of a row
  int64_t sa, sb;          // bytes of a matrix
  int32_t m, n;            // padded sides of the output
  int32_t pieces, per;     // of the reduction, of a slice
  int32_t slices;
  uint32_t tm, tn;
  uint32_t tiles;          // of a matrix
  float* part;             // slices: [batch][slice][tile][quad][thread] of four sums
  float unit;              // of the sum
  // outputs
  uint8_t *rowop, *colop;  // operand and (GRAM, POLY: the same) its transpose
  int64_t ldr, ldc, sr, sc;
  const uint8_t* old;      // POLY: cold times this joins (and cold2 old2, nullable); STEP, LAST: X
  const uint8_t* old2;     //   (its high part); in rowop's layout
  float cold, cold2;       // (with the units of what they multiply)
  float* diag;             // one part: POLY writes a + B_ii, STEP reads it, [rp] a matrix
  float ca;                // a, or a group's q
  float uout;              // unit of the operands written
  uint16_t* xlo;           // one part: X's low part
  int32_t R, C, rp;
  bool diag_cols;          // the diagonal goes by column (tall)
  void* out;
  float* w;
  float alpha, keep;
};

enum { GRAM, POLY, STEP, LAST };

template <int KIND>
__device__ __forceinline__ void mm_tile(const MmArgs& g, uint32_t id, uint32_t* im, uint32_t* in) {
  if (KIND == GRAM || KIND == POLY)
    tri_tile_of(id, g.tm, 8, im, in);
  else
    tile_of(id, g.tm, g.tn, 8, im, in);
}

// What a wave needs from memory for its sums at 16 FM rows from i0 by 32 columns from
// j0 (a lane: rows i0 + 16 fi + lane % 16, columns j0 + 8 (lane / 16) ..), all of it
// requested before the first is used.
template <int FM>
struct Old {
  uint4 hi[FM], lo[FM];
  float w[FM][8], dg[FM], dc[8];
};
template <Prod P, int KIND, bool MUON, int FM>
__device__ __forceinline__ void fetch_old(const MmArgs& g, int64_t b, int64_t i0, int64_t j0, Old<FM>& o) {
  constexpr bool ONE = P == Prod::F16, XSTEP = KIND == STEP || KIND == LAST;
  const int lane = threadIdx.x & 63;
  const int64_t j = j0 + (lane >> 4) * 8, i1 = i0 + (lane & 15);
  const bool in_n = j < g.n;
#pragma unroll
  for (int fi = 0; fi < FM; ++fi) {
    const int64_t i = i1 + fi * 16;
    o.hi[fi] = o.lo[fi] = make_uint4(0, 0, 0, 0);
    o.dg[fi] = 0.f;
    if (i >= g.m || !in_n) continue;
    if (KIND == POLY || XSTEP) {
      const uint4* d = (const uint4*)(g.old + b * g.sr + i * g.ldr + op_off<P>(j));
      o.hi[fi] = d[0];
      if (!ONE) o.lo[fi] = d[4];
      if (XSTEP && ONE) o.lo[fi] = *(const uint4*)(g.xlo + (b * g.m + i) * (int64_t)g.n + j);
    }
    if (XSTEP && ONE && !g.diag_cols) o.dg[fi] = g.diag[b * g.rp + i];
    if (KIND == LAST && MUON && i < g.R && j < g.C)
      load_n<DFP_F32, 8>(g.w + (b * g.R + i) * g.C + j, g.C - j, o.w[fi]);
  }
#pragma unroll
  for (int r = 0; r < 8; ++r) o.dc[r] = 0.f;
  if (XSTEP && ONE && g.diag_cols && in_n) load_n<DFP_F32, 8>(g.diag + b * g.rp + j, 8, o.dc);
}

// What becomes of those sums.  The transposed operand
// goes through LDS (`lds`: 32 columns of 16 FM + 8 numbers, this wave's own) so that it
// is stored in 16-byte runs too: stored from the lanes, two bytes at a time,
// 2048 x 8192's STEP took 217 us.
template <Prod P, int KIND, int T, bool MUON, int FM>
__device__ __forceinline__ void finish(const MmArgs& g, int64_t b, int64_t i0, int64_t j0, bool mirror, uint16_t* lds,
                                       float (&s)[FM][8], Old<FM>& o) {
  constexpr int kRows = 16 * FM, kStride = kRows + 8;
  constexpr bool ONE = P == Prod::F16, XSTEP = KIND == STEP || KIND == LAST;
  const int lane = threadIdx.x & 63;
  const int64_t j = j0 + (lane >> 4) * 8, i1 = i0 + (lane & 15);
  const bool in_n = j < g.n;
#pragma unroll
  for (int fi = 0; fi < FM; ++fi) {
    const int64_t i = i1 + fi * 16;
    float(&v)[8] = s[fi];
    if (i >= g.m || !in_n) continue;
#pragma unroll
    for (int r = 0; r < 8; ++r) v[r] *= g.unit;
    float x[8];
    if (KIND == POLY || XSTEP) unpack8(o.hi[fi], o.lo[fi], x);
    if (KIND == POLY && !ONE && g.old2) {
      const uint4* d = (const uint4*)(g.old2 + b * g.sr + i * g.ldr + op_off<P>(j));
      float y[8];
      unpack8(d[0], d[4], y);
#pragma unroll
      for (int r = 0; r < 8; ++r) v[r] = fmaf(g.cold2, y[r], v[r]);
    }
    if (KIND == POLY) {
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        v[r] = fmaf(g.cold, x[r], v[r]);
        if (ONE && i == j + r) {
          g.diag[b * g.rp + i] = g.ca + v[r];
          v[r] = 0.f;
        }
      }
    }
    if (XSTEP) {
#pragma unroll
      for (int r = 0; r < 8; ++r)
        v[r] = fmaf(ONE ? (g.diag_cols ? o.dc[r] : o.dg[fi]) : g.ca, x[r] * (1.f / (1 << kUnitX)), v[r]);
    }
    if (KIND == LAST) {
      if (i >= g.R || j >= g.C) continue;
      const int64_t at = (b * g.R + i) * g.C + j;
      if (MUON) {
#pragma unroll
        for (int r = 0; r < 8; ++r) o.w[fi][r] = fmaf(-g.alpha, v[r], g.keep * o.w[fi][r]);
        store_n<DFP_F32, 8>(g.w + at, g.C - j, o.w[fi]);
      } else {
        store_n<T, 8>((typename Elem<T>::type*)g.out + at, g.C - j, v);
      }
      continue;
    }
#pragma unroll
    for (int r = 0; r < 8; ++r) v[r] *= g.uout;
    put8<P>(g.rowop + b * g.sr + i * g.ldr, j, v);
    if (KIND == STEP && ONE) *(uint4*)(g.xlo + (b * g.m + i) * (int64_t)g.n + j) = pack8_low(v);
  }
  if (KIND == LAST || !mirror) return;
  // (g.m and g.n are multiples of 64: runs of eight are in or out as a whole)
#pragma unroll
  for (int part = 0; part < (P == Prod::F16X2 ? 2 : 1); ++part) {
#pragma unroll
    for (int fi = 0; fi < FM; ++fi)
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        const _Float16 hi = (_Float16)s[fi][r];
        lds[((lane >> 4) * 8 + r) * kStride + fi * 16 + (lane & 15)] =
            h_bits(part ? (_Float16)(s[fi][r] - (float)hi) : hi);
      }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int k = 0; k < kRows / 16; ++k) {
      const int c = (k * 64 + lane) / (kRows / 8), q = (k * 64 + lane) % (kRows / 8) * 8;
      const uint4 d = *(const uint4*)(lds + c * kStride + q);
      if (j0 + c < g.n && i0 + q < g.m)
        *(uint4*)(g.colop + b * g.sc + (j0 + c) * g.ldc + op_off<P>(i0 + q) + part * 64) = d;
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// Bound by the matrix cores where a CU has many pieces (2048 x 8192, two parts: Gram
// product 107 us, step 194 us, 1060 TFLOP/s of f16, a product of the small side 35 us);
// small ones by the launch, the first loads and the stores, 4 to 5 us, and the tiles'
// bytes from L2, about 60 KB a microsecond and CU (12 of 512 x 512, one part: 7.5 us,
// the step, whose three arrays are 46 MB in and out, 13.3).
template <Prod P, int KIND, int T, bool MUON, bool SLICED, class Q>
__global__ __launch_bounds__(Q::kThreads, 2) void k_mm(MmArgs g) {
  typedef typename Q::template Tile<P> Tile;
  constexpr int TM = Q::TM, TN = Q::TN, WM = Q::WM, WN = Q::WN;
  // matrices, their slices and those' tiles in order: an XCD's workgroups read few rows
  // (12 of 512 x 512 dealt out one by one: every XCD reads every matrix)
  const uint32_t id = xcd_order(blockIdx.x, gridDim.x), sl = id / g.tiles, tile = id - sl * g.tiles;
  const int64_t b = SLICED ? sl / g.slices : sl;
  const int32_t slice = SLICED ? sl % g.slices : 0;
  uint32_t im, in;
  mm_tile<KIND>(g, tile, &im, &in);
  const int32_t p0 = slice * g.per, pieces = SLICED ? min(g.per, g.pieces - p0) : g.pieces;
  const int64_t i0 = (int64_t)im * TM, j0 = (int64_t)in * TN, at = (int64_t)p0 * kPiece;
  const int wave = threadIdx.x >> 6;
  const int64_t iw = i0 + (wave / WN) * (TM / WM), jw = j0 + (wave % WN) * (TN / WN);
  // of a small tile, what joins its sums is under way from the start (12 updates of
  // 512 x 512 BF16 139.6 us without, 134.6 so; 1024 x 1024 FP32 184 and 177)
  constexpr bool EARLY = !SLICED && Tile::FN == 2;
  Old<Tile::FM> old;
  if (EARLY && threadIdx.x < Tile::kThreads) fetch_old<P, KIND, MUON>(g, b, iw, jw, old);
  mv4f acc[Tile::FM][Tile::FN];
  Tile::run(g.a + b * g.sa + i0 * g.lda + at, g.lda, (int32_t)(g.m - i0), g.b + b * g.sb + j0 * g.ldb + at, g.ldb,
            (int32_t)(g.n - j0), pieces, acc);
  if (!SLICED) __syncthreads();  // all waves are done with the stages
  if (threadIdx.x >= Tile::kThreads) return;
  if (SLICED) {
    mv4f* d = (mv4f*)g.part + (int64_t)id * (TM * TN / 4) + threadIdx.x;
#pragma unroll
    for (int j = 0; j < Tile::FN; ++j)
#pragma unroll
      for (int i = 0; i < Tile::FM; ++i) d[(j * Tile::FM + i) * Tile::kThreads] = acc[i][j];
    return;
  }
  uint16_t* lds = (uint16_t*)(Tile::template stage<0>() + wave * (Tile::kStage / (WM * WN)));
  static_assert(32 * (16 * Tile::FM + 8) * 2 <= Tile::kStage / (WM * WN), "a wave's part of a stage");
#pragma unroll
  for (int j = 0; j < Tile::FN; j += 2) {
    float s[Tile::FM][8];
#pragma unroll
    for (int i = 0; i < Tile::FM; ++i)
#pragma unroll
      for (int r = 0; r < 8; ++r) s[i][r] = acc[i][j + (r >> 2)][r & 3];
    if (!EARLY) fetch_old<P, KIND, MUON>(g, b, iw, jw + j * 16, old);
    finish<P, KIND, T, MUON, Tile::FM>(g, b, iw, jw + j * 16, KIND == STEP || im != in, lds, s, old);
  }
}

// The slices of a tile added up in their order, then as above: workgroups of a tile's
// threads by one pair of fragment columns.  5.0 us for 8 slices of 384 x 384: the launch
// and two trips to memory.
template <Prod P, class Q>
__global__ __launch_bounds__(64 * Q::WM * Q::WN) void k_sum(MmArgs g) {
  typedef typename Q::template Tile<P> Tile;
  constexpr int TM = Q::TM, TN = Q::TN, WM = Q::WM, WN = Q::WN;
  constexpr int FM = Tile::FM, FN = Tile::FN;
  __shared__ __align__(16) uint16_t lds[WM * WN][32 * (16 * FM + 8)];
  const int64_t b = blockIdx.y;
  const uint32_t id = blockIdx.x / (FN / 2), j = blockIdx.x % (FN / 2) * 2;
  uint32_t im, in;
  mm_tile<GRAM>(g, id, &im, &in);
  const int64_t stride = (int64_t)g.tiles * (TM * TN / 4);  // of a slice
  const mv4f* d = (const mv4f*)g.part + b * g.slices * stride + (int64_t)id * (TM * TN / 4) + threadIdx.x;
  float s[FM][8] = {};
  constexpr int U = FM > 2 ? 4 : 8;  // slices in flight
  for (int32_t k = 0; k < g.slices; k += U) {
    mv4f v[U][FM][2];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h)
          v[u][i][h] = d[min(k + u, g.slices - 1) * stride + ((j + h) * FM + i) * Tile::kThreads];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (k + u < g.slices) {
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
          for (int r = 0; r < 8; ++r) s[i][r] += v[u][i][r >> 2][r & 3];
      }
  }
  const int wave = threadIdx.x >> 6;
  Old<FM> none;
  finish<P, GRAM, 0, false, FM>(g, b, (int64_t)im * TM + (wave / WN) * (TM / WM),
                                (int64_t)in * TN + (wave % WN) * (TN / WN) + j * 16, im != in, lds[wave], s, none);
}

template <Prod P, int KIND, int T, bool MUON>
dfp_status launch_mm(int32_t id, const MmPlan& p, int32_t batch, MmArgs& g, hipStream_t st) {
  const TileKind& kind = kTileKinds[p.kind];
  g.tm = (uint32_t)((g.m + kind.tm - 1) / kind.tm);
  g.tn = (uint32_t)((g.n + kind.tn - 1) / kind.tn);
  g.per = p.per;
  g.slices = p.slices;
  constexpr bool SYM = KIND == GRAM || KIND == POLY;
  g.tiles = SYM ? g.tm * (g.tm + 1) / 2 : g.tm * g.tn;
  const uint32_t wgs = g.tiles * (uint32_t)batch;
  return with_tile(p.kind, [&](auto shape) -> dfp_status {
    typedef decltype(shape) Q;
    if constexpr (SYM && (Q::TM != Q::TN || (P == Prod::F16X2 && Q::TM == 96 && Q::KG == 1))) {
      return DFP_ERR_PARAM;  // (has_triangle: no plan has it)
    } else {
      if constexpr (KIND == GRAM) {
        if (p.slices > 1) {
          DFP_LAUNCH(id, (k_mm<P, KIND, T, MUON, true, Q>), dim3(wgs * p.slices), dim3(Q::kThreads), 0, st, g);
          DFP_LAUNCH(id, (k_sum<P, Q>), dim3(g.tiles * (Q::TN / Q::WN / 32), (unsigned)batch),
                     dim3(64 * Q::WM * Q::WN), 0, st, g);
          return DFP_OK;
        }
      }
      DFP_LAUNCH(id, (k_mm<P, KIND, T, MUON, false, Q>), dim3(wgs), dim3(Q::kThreads), 0, st, g);
      return DFP_OK;
    }
  });
}

// Largest |a + b s + c s^2| on [0, 1]: at an end or at the vertex.
double most_of(double a, double b, double c) {
  double m = std::max(std::fabs(a), std::fabs(a + b + c));
  const double s = c != 0. ? -b / (2. * c) : 0.;
  if (s > 0. && s < 1.) m = std::max(m, std::fabs(a + s * (b + s * c)));
  return m;
}

// Largest unit, 2^12 at most, that keeps an operand of up to `most` at 32768 or less.
float unit_for(double most) {
  int s = 12;
  while (s > 0 && most * (double)(1 << s) > 32768.) --s;
  return (float)(1 << s);
}

// Unit of B = b A + c A A.  Up to A = 2: by its terms.  From there to 16: by its terms, or,
// since |a + B| sqrt(A) <= 4 after the step, |B| <= |a| + 4 / sqrt(2).
float unit_b(double a, double b, double c) {
  a = std::fabs(a), b = std::fabs(b), c = std::fabs(c);
  return unit_for(std::max(2. * b + 4. * c, std::min(16. * b + 256. * c, a + 2.83)));
}

template <int T, bool MUON, Prod P>
dfp_status run(const dfp_ortho_desc& d, const Source<T>& src, void* out, float* w, float alpha, float keep, void* ws,
               hipStream_t st) {
  constexpr bool SPLIT = P == Prod::F16X2;
  constexpr int64_t kPerPiece = SPLIT ? 32 : 64;  // elements of a piece
  const Plan p = make_plan(d, SPLIT);
  uint8_t* base = (uint8_t*)ws;
  uint16_t* xlo = (uint16_t*)(base + p.xlo);
  uint8_t *gram = base + p.gram, *aa = base + p.aa, *bb = base + p.bb;
  uint8_t* step[2] = {base + p.step0, base + p.step1};
  double* part = (double*)(base + p.norm);
  const unsigned nb = (unsigned)d.batch;
  const int64_t n = p.R * p.C;
  const int32_t parts = (int32_t)std::min<int64_t>(n < (1 << 23) ? kBlock : kNormParts, (n + kBlock * 16 - 1) / (kBlock * 16));
  DFP_LAUNCH(K_ORTHO_NORM, (k_norm<T, MUON>), dim3((unsigned)parts, nb), dim3(kBlock), 0, st, src, n, part);
  // gram: the longer side contiguous
  uint8_t* rowop = p.tall ? step[0] : gram;
  uint8_t* colop = p.tall ? gram : step[0];
  DFP_LAUNCH(K_ORTHO_PACK, (k_pack<T, MUON, P>), dim3((unsigned)(p.Rp / 64 * (p.Cp / 64)), nb), dim3(kBlock), 0, st,
             src, p.R, p.C, p.Rp, p.Cp, part, parts, d.eps, xlo, rowop, colop);
  const int64_t longer = p.tall ? p.Rp : p.Cp;
  const int64_t sx = p.Rp * p.Cp * p.e, ss = p.rp * p.rp * p.e;
  constexpr float kInvX = 1.f / (1 << kUnitX), kInvA = 1.f / (1 << kUnitA);
  // C = A B of the small side, symmetric: C = unit A B + c X [+ c2 Y], times uout
  uint8_t *pa = base + p.pa, *qq[2] = {base + p.qq0, base + p.qq1};
  MmArgs g{};
  auto small = [&](const uint8_t* a, const uint8_t* b, uint8_t* to, float unit, const uint8_t* x, float c, float uout,
                   const uint8_t* y = nullptr, float c2 = 0.f) -> dfp_status {
    g.a = a, g.b = b;
    g.lda = g.ldb = g.ldr = g.ldc = p.rp * p.e;
    g.sa = g.sb = g.sr = g.sc = ss;
    g.m = g.n = (int32_t)p.rp;
    g.pieces = (int32_t)(p.rp / kPerPiece);
    g.unit = unit;
    g.old = x, g.cold = c;
    g.old2 = y, g.cold2 = c2;
    g.uout = uout;
    g.rowop = g.colop = to;
    return launch_mm<P, POLY, 0, false>(K_ORTHO_POLY, p.mm.poly, d.batch, g, st);
  };
  dfp_status rc;
  for (int32_t s = 0, turn = 0; s < d.steps; ++turn) {
    g = MmArgs{};
    g.rp = (int32_t)p.rp;
    g.diag = (float*)(base + p.diag);
    g.part = (float*)(base + p.slices);
    // A = X X^T
    g.a = g.b = gram;
    g.lda = g.ldb = longer * p.e;
    g.sa = g.sb = sx;
    g.m = g.n = (int32_t)p.rp;
    g.pieces = (int32_t)(longer / kPerPiece);
    g.unit = kInvX * kInvX;
    g.uout = (float)(1 << kUnitA);
    g.rowop = g.colop = aa;
    g.ldr = g.ldc = p.rp * p.e;
    g.sr = g.sc = ss;
    if ((rc = launch_mm<P, GRAM, 0, false>(K_ORTHO_GRAM, p.mm.gram, d.batch, g, st)) != DFP_OK) return rc;
    // Q = B = b A + c A A, and what further iterations make of it; X = q X + Q X in the end
    uint8_t* q = bb;
    float uq = 1.f;
    double qa = 1., grown = 1., top = 1.;
    for (int32_t k = 0;; ++k, ++s) {
      const float ca = d.coef[s][0], cb = d.coef[s][1], cc = d.coef[s][2];
      const float ub = unit_b(ca, cb, cc);
      const double most = most_of(ca, cb, cc);
      uint8_t* to = k == 0 && MUON && p.mm.grouped ? qq[0] : bb;
      g.ca = ca;
      if ((rc = small(aa, aa, to, cc * kInvA * kInvA, aa, cb * kInvA, ub)) != DFP_OK) return rc;
      if (k == 0) {
        q = to, uq = ub;
      } else {
        // |P_2 P_1|: to the first X of a singular value above 1 the product of the steps'
        // largest on [0, 1], and from there 4, since no X ends above it
        const float un = unit_for(std::max(std::sqrt(grown) * most, 4. * top) + std::fabs(qa * ca));
        if ((rc = small(bb, q, qq[k & 1], 1.f / (ub * uq), q, ca / uq, un, bb, (float)qa / ub)) != DFP_OK) return rc;
        q = qq[k & 1], uq = un;
      }
      qa *= ca;
      grown *= most * most;
      top = std::max(top, std::sqrt(grown));
      if (!MUON || !p.mm.grouped || s + 1 >= d.steps || grown > 150.) break;
      if (grown * (std::fabs(d.coef[s + 1][1]) + 2. * std::fabs(d.coef[s + 1][2])) > 1600.) break;
      // A = P A P
      const float ua = (float)(1 << kUnitA);
      if ((rc = small(to, aa, pa, kInvA / ub, aa, ca * kInvA, ua)) != DFP_OK) return rc;
      if ((rc = small(to, pa, aa, kInvA / ub, pa, ca * kInvA, ua)) != DFP_OK) return rc;
    }
    ++s;
    // X = q X + Q X, in the caller's orientation: rows of Q by rows of X^T, or rows of X by rows of Q
    uint8_t *from = step[turn & 1], *to = step[(turn + 1) & 1];
    g.a = p.tall ? from : q;
    g.b = p.tall ? q : from;
    g.sa = p.tall ? sx : ss;
    g.sb = p.tall ? ss : sx;
    g.m = (int32_t)p.Rp, g.n = (int32_t)p.Cp;
    g.unit = kInvX / uq;
    g.uout = (float)(1 << kUnitX);
    g.rowop = p.tall ? to : gram;
    g.colop = p.tall ? gram : to;
    g.old = p.tall ? from : gram;
    g.ldr = p.Cp * p.e, g.ldc = p.Rp * p.e;
    g.sr = g.sc = sx;
    g.ca = (float)qa;
    g.xlo = xlo;
    g.R = (int32_t)p.R, g.C = (int32_t)p.C;
    g.diag_cols = p.tall;
    g.out = out;
    g.w = w;
    g.alpha = alpha, g.keep = keep;
    if (s < d.steps)
      rc = launch_mm<P, STEP, 0, false>(K_ORTHO_STEP, p.mm.step, d.batch, g, st);
    else
      rc = launch_mm<P, LAST, MUON ? DFP_F32 : T, MUON>(K_ORTHO_STEP, p.mm.step, d.batch, g, st);
    if (rc != DFP_OK) return rc;
  }
  return DFP_OK;
}

}  // namespace

// (either precision: one descriptor serves both calls)
size_t ortho_workspace_bytes(const dfp_ortho_desc& d) {
  return (size_t)std::max(make_plan(d, true).bytes, make_plan(d, false).bytes);
}

dfp_status launch_orthogonalize(const dfp_ortho_desc& d, const void* x, void* out, void* ws, hipStream_t st) {
  return with_type(d.type, [&](auto tc) -> dfp_status {
    constexpr int T = decltype(tc)::value;
    constexpr Prod P = T == DFP_BF16 ? Prod::F16 : Prod::F16X2;
    const Source<T> s{(const typename Elem<T>::type*)x, nullptr, 0.f, false};
    return run<T, false, P>(d, s, out, nullptr, 0.f, 0.f, ws, st);
  });
}

dfp_status launch_muon(const dfp_ortho_desc& d, float alpha, float keep, float mu, bool nesterov, float* w, float* v,
                       const void* dw, void* ws, hipStream_t st) {
  return with_type(d.type, [&](auto tc) -> dfp_status {
    constexpr int T = decltype(tc)::value;
    const Source<T> s{(const typename Elem<T>::type*)dw, v, mu, nesterov};
    return run<T, true, Prod::F16X2>(d, s, nullptr, w, alpha, keep, ws, st);
  });
}

}  // namespace dfp
