// Orthogonalised updates (see dfp.h): X = U / (|U| + eps), then steps of
//   A = X X^T, B = b A + c A A, X = a X + B X
// with the smaller side first (X^T X and X B where rows > cols).
//
// X [R][C] lives in FP32 in the caller's orientation.  The products read f16
// operands in the layout of mma_tile.h: `gram` is X (or X^T where R > C) with its
// longer side contiguous, `step` the other of the two; both are written by the
// kernel that makes X.  All sides are padded to 128 with zeros, which every step
// keeps zero.  A and B are symmetric: only tiles on and above the diagonal are
// computed and each is stored twice.  B's diagonal, the largest entries of its
// rows, stays out of the f16 operand and joins in FP32: X = (a + B_ii) X + B' X.
//
// Units: X in 2^-12, A in 2^-10, B in 2^-sb so that |b A + c A A| <= 32768 in it
// for singular values up to sqrt(2).
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
constexpr int kNormParts = 256;

struct Plan {
  bool tall;             // rows > cols
  int64_t R, C, Rp, Cp;  // the matrix, padded
  int64_t r, rp;         // the smaller side, padded
  int64_t e;             // bytes of an operand element
  int64_t x32, gram, step0, step1, aa, bb, diag, norm, bytes;  // offsets, total
};

Plan make_plan(const dfp_ortho_desc& d, bool split) {
  Plan p;
  p.R = d.rows;
  p.C = d.cols;
  p.tall = d.rows > d.cols;
  p.Rp = (p.R + 127) / 128 * 128;
  p.Cp = (p.C + 127) / 128 * 128;
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
  p.x32 = take(n * 4);
  p.gram = take(n * p.e);
  p.step0 = take(n * p.e);
  p.step1 = take(n * p.e);
  p.aa = take(s * p.e);
  p.bb = take(s * p.e);
  p.diag = take(p.rp * d.batch * 4);
  p.norm = take((int64_t)kNormParts * d.batch * 8);
  p.bytes = at;
  return p;
}

bool splits(int32_t type) { return type != DFP_BF16; }

// ---------------------------------------------------------------- operands
// Byte offset of element k of a row.
template <Prod P>
__device__ __forceinline__ int64_t op_off(int64_t k) {
  return P == Prod::F16X2 ? (k >> 5) * 128 + (k & 31) * 2 : k * 2;
}
__device__ __forceinline__ uint16_t h_bits(_Float16 h) { return __builtin_bit_cast(uint16_t, h); }
__device__ __forceinline__ float h_val(uint32_t b) { return (float)__builtin_bit_cast(_Float16, (uint16_t)b); }

// v (in units already) to element k of the row at p.
template <Prod P>
__device__ __forceinline__ void put1(uint8_t* p, int64_t k, float v) {
  uint16_t* d = (uint16_t*)(p + op_off<P>(k));
  const _Float16 hi = (_Float16)v;
  d[0] = h_bits(hi);
  if (P == Prod::F16X2) d[32] = h_bits((_Float16)(v - (float)hi));
}
// Four elements k .. k + 3, k a multiple of 4.
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
template <Prod P>
__device__ __forceinline__ void put8(uint8_t* p, int64_t k, const float (&v)[8]) {
  uint32_t hi[4], lo[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const _Float16 a = (_Float16)v[2 * i], b = (_Float16)v[2 * i + 1];
    hi[i] = h_bits(a) | (uint32_t)h_bits(b) << 16;
    lo[i] = h_bits((_Float16)(v[2 * i] - (float)a)) | (uint32_t)h_bits((_Float16)(v[2 * i + 1] - (float)b)) << 16;
  }
  uint4* d = (uint4*)(p + op_off<P>(k));
  d[0] = make_uint4(hi[0], hi[1], hi[2], hi[3]);
  if (P == Prod::F16X2) d[4] = make_uint4(lo[0], lo[1], lo[2], lo[3]);
}
template <Prod P>
__device__ __forceinline__ void get8(const uint8_t* p, int64_t k, float (&v)[8]) {
  const uint4* d = (const uint4*)(p + op_off<P>(k));
  const uint4 h = d[0];
  const uint32_t hw[4] = {h.x, h.y, h.z, h.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) v[2 * i] = h_val(hw[i]), v[2 * i + 1] = h_val(hw[i] >> 16);
  if (P == Prod::F16X2) {
    const uint4 l = d[4];
    const uint32_t lw[4] = {l.x, l.y, l.z, l.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) v[2 * i] += h_val(lw[i]), v[2 * i + 1] += h_val(lw[i] >> 16);
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
template <int T, bool MUON>
__device__ __forceinline__ void direction(const Source<T>& s, int64_t at, int64_t have, float (&u)[4]) {
  load_n<T, 4>(s.x + at, have, u);
  if (MUON) {
    float v[4];
    load_n<DFP_F32, 4>(s.v + at, have, v);
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = s.nesterov ? fmaf(s.mu, v[i], u[i]) : v[i];
  }
}

// Momentum update and partial sums of u^2 (in 64 bits), kNormParts a matrix.
template <int T, bool MUON>
__global__ __launch_bounds__(kBlock) void k_norm(Source<T> s, int64_t n, double* __restrict__ part) {
  __shared__ double red[kBlock / 64];
  const int64_t base = (int64_t)blockIdx.y * n;
  double sum = 0.;
  for (int64_t i = ((int64_t)blockIdx.x * kBlock + threadIdx.x) * 4; i < n; i += (int64_t)kNormParts * kBlock * 4) {
    float u[4];
    if (MUON) {
      float g[4], v[4];
      load_n<T, 4>(s.x + base + i, n - i, g);
      load_n<DFP_F32, 4>(s.v + base + i, n - i, v);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        v[j] = fmaf(s.mu, v[j], g[j]);
        u[j] = s.nesterov ? fmaf(s.mu, v[j], g[j]) : v[j];
      }
      store_n<DFP_F32, 4>(s.v + base + i, n - i, v);
    } else {
      load_n<T, 4>(s.x + base + i, n - i, u);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) sum += (double)u[j] * (double)u[j];
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x == 0) part[(int64_t)blockIdx.y * kNormParts + blockIdx.x] = (red[0] + red[1]) + (red[2] + red[3]);
}

// X = u / (|u| + eps): FP32 and both operands, 64 x 64 tiles of the padded matrix.
template <int T, bool MUON, Prod P>
__global__ __launch_bounds__(kBlock) void k_pack(Source<T> s, int64_t R, int64_t C, int64_t Rp, int64_t Cp,
                                                 const double* __restrict__ part, float eps, float* __restrict__ x32,
                                                 uint8_t* __restrict__ rowop, uint8_t* __restrict__ colop) {
  __shared__ float tile[64][65];
  __shared__ double red[kBlock / 64];
  const int64_t b = blockIdx.y;
  double sum = part[b * kNormParts + threadIdx.x];
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = sum;
  __syncthreads();
  const double nrm = sqrt((red[0] + red[1]) + (red[2] + red[3]));
  const double inv = isfinite(nrm) ? 1. / (nrm + (double)eps) : (double)__uint_as_float(0x7fc00000u);
  const int64_t ct = Cp / 64, r0 = blockIdx.x / ct * 64, c0 = blockIdx.x % ct * 64;
  const int cc = (threadIdx.x & 15) * 4;
  const int64_t pbytes = Rp * Cp * (P == Prod::F16X2 ? 4 : 2);
  constexpr int64_t e = P == Prod::F16X2 ? 4 : 2;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int rr = (threadIdx.x >> 4) + i * 16;
    const int64_t r = r0 + rr, c = c0 + cc;
    float u[4] = {0.f, 0.f, 0.f, 0.f};
    if (r < R && c < C) direction<T, MUON>(s, (b * R + r) * C + c, C - c, u);
#pragma unroll
    for (int j = 0; j < 4; ++j) u[j] = r < R && c + j < C ? (float)((double)u[j] * inv) : 0.f;
    *(float4*)(x32 + (b * Rp + r) * Cp + c) = make_float4(u[0], u[1], u[2], u[3]);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      u[j] *= (float)(1 << kUnitX);
      tile[rr][cc + j] = u[j];
    }
    put4<P>(rowop + b * pbytes + r * Cp * e, c, u);
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int rr = (threadIdx.x >> 4) + i * 16;
    const float u[4] = {tile[cc][rr], tile[cc + 1][rr], tile[cc + 2][rr], tile[cc + 3][rr]};
    put4<P>(colop + b * pbytes + (c0 + rr) * Rp * e, r0 + cc, u);
  }
}

// ---------------------------------------------------------------- products
struct MmArgs {
  const uint8_t *a, *b;    // operands, of one batch element
  int64_t lda, ldb;        // bytes of a row
  int64_t sa, sb;          // bytes of a matrix
  int32_t m, n;            // padded sides of the output
  int32_t pieces;
  uint32_t tm, tn;
  float unit;              // of the sum
  // outputs
  uint8_t *rowop, *colop;  // operand and (GRAM / POLY: the same) its transpose
  int64_t ldr, ldc, sr, sc;
  const uint8_t* aa;       // POLY: A
  float* diag;             // POLY writes, STEP reads, [rp] a matrix
  float cb, cc, ca;        // coefficients
  float uout;              // unit of the operands written
  float* x32;
  int32_t R, C, rp;
  bool diag_cols;          // the diagonal goes by column (tall)
  void* out;
  float* w;
  float alpha, keep;
};

enum { GRAM, POLY, STEP, LAST };

// Tile (i, j), i <= j, of a triangle of t tiles a side.
__device__ __forceinline__ void tri_tile(uint32_t id, uint32_t t, uint32_t* i, uint32_t* j) {
  uint32_t row = 0, left = t;
  while (id >= left) {
    id -= left;
    ++row;
    --left;
  }
  *i = row;
  *j = row + id;
}

template <Prod P, int KIND, int T, bool MUON, int TM, int TN, int WM, int WN, int S>
__global__ __launch_bounds__(64 * WM * WN, 2) void k_mm(MmArgs g) {
  typedef MmaTile<P, TM, TN, WM, WN, S> Tile;
  const int64_t b = blockIdx.y;
  uint32_t im, in;
  if (KIND == GRAM || KIND == POLY)
    tri_tile(blockIdx.x, g.tm, &im, &in);
  else
    tile_of(blockIdx.x, g.tm, g.tn, 8, &im, &in);
  const int64_t i0 = (int64_t)im * TM, j0 = (int64_t)in * TN;
  mv4f acc[Tile::FM][Tile::FN];
  Tile::run(g.a + b * g.sa + i0 * g.lda, g.lda, (int32_t)(g.m - i0), g.b + b * g.sb + j0 * g.ldb, g.ldb,
            (int32_t)(g.n - j0), g.pieces, acc);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t i1 = i0 + (wave / WN) * (TM / WM) + (lane & 15);
  const int64_t j1 = j0 + (wave % WN) * (TN / WN) + (lane >> 4) * 8;
#pragma unroll
  for (int fj = 0; fj < Tile::FN; fj += 2)
#pragma unroll
    for (int fi = 0; fi < Tile::FM; ++fi) {
      const int64_t i = i1 + fi * 16, j = j1 + fj * 16;
      if (i >= g.m || j >= g.n) continue;
      float v[8];
#pragma unroll
      for (int r = 0; r < 8; ++r) v[r] = acc[fi][fj + (r >> 2)][r & 3] * g.unit;
      if (KIND == POLY) {
        float a[8];
        get8<P>(g.aa + b * g.sr + i * g.ldr, j, a);
#pragma unroll
        for (int r = 0; r < 8; ++r) {
          v[r] = fmaf(g.cc, v[r], g.cb * (a[r] * (1.f / (1 << kUnitA))));
          if (i == j + r) {
            g.diag[b * g.rp + i] = v[r];
            v[r] = 0.f;
          }
        }
      }
      if (KIND == STEP || KIND == LAST) {
        float* px = g.x32 + (b * g.m + i) * (int64_t)g.n + j;
        const float4 x0 = *(const float4*)px, x1 = *(const float4*)(px + 4);
        const float xs[8] = {x0.x, x0.y, x0.z, x0.w, x1.x, x1.y, x1.z, x1.w};
#pragma unroll
        for (int r = 0; r < 8; ++r) v[r] = fmaf(g.ca + g.diag[b * g.rp + (g.diag_cols ? j + r : i)], xs[r], v[r]);
        if (KIND == STEP) {
          *(float4*)px = make_float4(v[0], v[1], v[2], v[3]);
          *(float4*)(px + 4) = make_float4(v[4], v[5], v[6], v[7]);
        }
      }
      if (KIND == LAST) {
        if (i >= g.R || j >= g.C) continue;
        const int64_t at = (b * g.R + i) * g.C + j;
        if (MUON) {
          float w[8];
          load_n<DFP_F32, 8>(g.w + at, g.C - j, w);
#pragma unroll
          for (int r = 0; r < 8; ++r) w[r] = fmaf(-g.alpha, v[r], g.keep * w[r]);
          store_n<DFP_F32, 8>(g.w + at, g.C - j, w);
        } else {
          store_n<T, 8>((typename Elem<T>::type*)g.out + at, g.C - j, v);
        }
        continue;
      }
#pragma unroll
      for (int r = 0; r < 8; ++r) v[r] *= g.uout;
      put8<P>(g.rowop + b * g.sr + i * g.ldr, j, v);
      if (KIND == STEP || im != in) {
#pragma unroll
        for (int r = 0; r < 8; ++r) put1<P>(g.colop + b * g.sc + (j + r) * g.ldc, i, v[r]);
      }
    }
}

// Largest unit of B that keeps |b A + c A A| at 32768 or less for |X| <= sqrt(2).
float unit_b(const float* coef) {
  const double most = std::fabs((double)coef[1]) * 2. + std::fabs((double)coef[2]) * 4.;
  int s = 12;
  while (s > 0 && most * (double)(1 << s) > 32768.) --s;
  return (float)(1 << s);
}

template <int T, bool MUON, Prod P>
dfp_status run(const dfp_ortho_desc& d, const Source<T>& src, void* out, float* w, float alpha, float keep, void* ws,
               hipStream_t st) {
  constexpr bool SPLIT = P == Prod::F16X2;
  constexpr int64_t kPerPiece = SPLIT ? 32 : 64;  // elements of a piece
  const Plan p = make_plan(d, SPLIT);
  uint8_t* base = (uint8_t*)ws;
  float* x32 = (float*)(base + p.x32);
  uint8_t *gram = base + p.gram, *aa = base + p.aa, *bb = base + p.bb;
  uint8_t* step[2] = {base + p.step0, base + p.step1};
  double* part = (double*)(base + p.norm);
  const unsigned nb = (unsigned)d.batch;
  DFP_LAUNCH(K_ORTHO_NORM, (k_norm<T, MUON>), dim3(kNormParts, nb), dim3(kBlock), 0, st, src, p.R * p.C, part);
  // gram: the longer side contiguous
  uint8_t* rowop = p.tall ? step[0] : gram;
  uint8_t* colop = p.tall ? gram : step[0];
  DFP_LAUNCH(K_ORTHO_PACK, (k_pack<T, MUON, P>), dim3((unsigned)(p.Rp / 64 * (p.Cp / 64)), nb), dim3(kBlock), 0, st,
             src, p.R, p.C, p.Rp, p.Cp, part, d.eps, x32, rowop, colop);
  const int64_t longer = p.tall ? p.Rp : p.Cp;
  const int64_t sx = p.Rp * p.Cp * p.e, ss = p.rp * p.rp * p.e;
  constexpr float kInvX = 1.f / (1 << kUnitX), kInvA = 1.f / (1 << kUnitA);
  constexpr int TM = 128, TN = 128;
  for (int32_t s = 0; s < d.steps; ++s) {
    const float ub = unit_b(d.coef[s]);
    const uint32_t ts = (uint32_t)(p.rp / TM);
    MmArgs g{};
    g.rp = (int32_t)p.rp;
    g.diag = (float*)(base + p.diag);
    g.ca = d.coef[s][0], g.cb = d.coef[s][1], g.cc = d.coef[s][2];
    // A = X X^T
    g.a = g.b = gram;
    g.lda = g.ldb = longer * p.e;
    g.sa = g.sb = sx;
    g.m = g.n = (int32_t)p.rp;
    g.pieces = (int32_t)(longer / kPerPiece);
    g.tm = g.tn = ts;
    g.unit = kInvX * kInvX;
    g.uout = (float)(1 << kUnitA);
    g.rowop = g.colop = aa;
    g.ldr = g.ldc = p.rp * p.e;
    g.sr = g.sc = ss;
    DFP_LAUNCH(K_ORTHO_GRAM, (k_mm<P, GRAM, 0, false, TM, TN, 2, 2, 2>), dim3(ts * (ts + 1) / 2, nb), dim3(256), 0, st, g);
    // B = b A + c A A
    g.a = g.b = g.aa = aa;
    g.lda = g.ldb = p.rp * p.e;
    g.sa = g.sb = ss;
    g.pieces = (int32_t)(p.rp / kPerPiece);
    g.unit = kInvA * kInvA;
    g.uout = ub;
    g.rowop = g.colop = bb;
    DFP_LAUNCH(K_ORTHO_POLY, (k_mm<P, POLY, 0, false, TM, TN, 2, 2, 2>), dim3(ts * (ts + 1) / 2, nb), dim3(256), 0, st, g);
    // X = a X + B X, in the caller's orientation: rows of B by rows of X^T, or rows of X by rows of B
    uint8_t *from = step[s & 1], *to = step[(s + 1) & 1];
    g.a = p.tall ? from : bb;
    g.b = p.tall ? bb : from;
    g.sa = p.tall ? sx : ss;
    g.sb = p.tall ? ss : sx;
    g.m = (int32_t)p.Rp, g.n = (int32_t)p.Cp;
    g.tm = (uint32_t)(p.Rp / TM), g.tn = (uint32_t)(p.Cp / TN);
    g.unit = kInvX / ub;
    g.uout = (float)(1 << kUnitX);
    g.rowop = p.tall ? to : gram;
    g.colop = p.tall ? gram : to;
    g.ldr = p.Cp * p.e, g.ldc = p.Rp * p.e;
    g.sr = g.sc = sx;
    g.x32 = x32;
    g.R = (int32_t)p.R, g.C = (int32_t)p.C;
    g.diag_cols = p.tall;
    g.out = out;
    g.w = w;
    g.alpha = alpha, g.keep = keep;
    const dim3 grid(g.tm * g.tn, nb);
    if (s + 1 < d.steps)
      DFP_LAUNCH(K_ORTHO_STEP, (k_mm<P, STEP, 0, false, TM, TN, 2, 2, 2>), grid, dim3(256), 0, st, g);
    else
      DFP_LAUNCH(K_ORTHO_STEP, (k_mm<P, LAST, T, MUON, TM, TN, 2, 2, 2>), grid, dim3(256), 0, st, g);
  }
  return DFP_OK;
}

}  // namespace

size_t ortho_workspace_bytes(const dfp_ortho_desc& d) { return (size_t)make_plan(d, true).bytes; }

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
