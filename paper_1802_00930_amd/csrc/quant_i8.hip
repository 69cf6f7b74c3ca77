// INT8 quantisation with one FP32 scale per row or column (see dfp.h), the
// operands of the INT8 linear layers.
//   rows      a row's workgroup (or wave) keeps the row in registers between its
//             maximum and its rounding: one read, one write
//   columns   over the tokens of a gradient: partial maxima of slices of the
//             rows, then the rounding into the transposed layout
// Both are bound by memory (a large copy runs at 4.92 TB/s): the exact rounding, a
// product, a fused difference and a test that it is the nearest, costs five operations
// an element, and only where the test fails the ones that mend it.  Stochastic rounding is
// bound by arithmetic: the exact rounding, a division and a Philox word an element.
#include <algorithm>
#include <type_traits>

#include "dfp_internal.h"
#include "dfp_round.h"
#include "dfp_types.h"
#include "i8_round.h"
#include "linear_i8.h"

#pragma clang fp contract(off)

namespace dfp {

namespace {

constexpr int kBlock = 256;

// Rows by groups of G threads (64: four rows a workgroup, 256: one), NV vectors of
// 8 elements a thread in registers; NV = 0: a row of any length, read twice.
// colw (nullable): every element is first multiplied by its column's weight.
// 8192 x 2048: BF16 12.1 to 13.7 us (4.2 to 3.7 TB/s), FP32 14.7 us (5.7 TB/s, a part of it
// from the memory-side cache); 16384 x 8192 BF16 72.6 to 83 us (5.5 to 4.9 TB/s).  Stochastic:
// 32.5, 32.4 and 198 us.
template <int T, int MODE, int G, int NV, bool WEIGHTED>
__global__ __launch_bounds__(kBlock) void k_rows_i8(const typename Elem<T>::type* __restrict__ src, int64_t rows,
                                                    int64_t cols, int64_t ld, const float* __restrict__ colw,
                                                    int8_t* __restrict__ q, float* __restrict__ scale, uint32_t k0,
                                                    uint32_t k1, uint32_t role) {
  __shared__ uint32_t red[kBlock / 64];
  const int t = threadIdx.x % G;
  const int64_t per = kBlock / G, nvec = ld / 8;
  // (every thread of a workgroup makes the same number of rounds)
  for (int64_t r0 = (int64_t)blockIdx.x * per; r0 < rows; r0 += (int64_t)gridDim.x * per) {
    const int64_t r = min(r0 + threadIdx.x / G, rows - 1);
    const bool mine = r0 + threadIdx.x / G < rows;
    const typename Elem<T>::type* x = src + r * cols;
    Raw<T, 8> raw[NV > 0 ? NV : 1];
    Raw<DFP_F32, 8> weight[NV > 0 && WEIGHTED ? NV : 1];
    auto fetch = [&](int64_t c, int i) {
      fetch_n<T, 8>(x + c, cols - c, raw[i]);
      if (WEIGHTED) fetch_n<DFP_F32, 8>(colw + c, cols - c, weight[i]);
    };
    auto number = [&](int i, float (&v)[8]) {
      up_n<T, 8>(raw[i], v);
      if (WEIGHTED) {
        float w[8];
        up_n<DFP_F32, 8>(weight[i], w);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= w[e];
      }
    };
    uint32_t mx = 0;
    auto maxof = [&](const float (&v)[8]) {
#pragma unroll
      for (int i = 0; i < 8; ++i) mx = max(mx, __float_as_uint(v[i]) & 0x7fffffffu);
    };
    float v[NV > 0 ? NV : 1][8];
    if constexpr (NV > 0) {
#pragma unroll
      for (int i = 0; i < NV; ++i) fetch(((int64_t)t + i * G) * 8, i);
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        number(i, v[i]);
        maxof(v[i]);
      }
    } else {
      for (int64_t c = t; c < nvec; c += G) {
        fetch(c * 8, 0);
        number(0, v[0]);
        maxof(v[0]);
      }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) mx = max(mx, (uint32_t)__shfl_xor((int)mx, o, 64));
    if constexpr (G > 64) {
      __syncthreads();
      if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = mx;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < kBlock / 64; ++w) mx = max(mx, red[w]);
    }
    const I8Scale k = i8_scale(mx);
    if (t == 0 && mine) scale[r] = k.s;
    if constexpr (NV > 0) {
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int64_t c = (int64_t)t + i * G;
        if (mine && c < nvec)
          *reinterpret_cast<uint2*>(q + r * ld + c * 8) = i8_round8<MODE>(v[i], k, r * cols + c * 8, k0, k1, role);
      }
    } else {
      for (int64_t c = t; c < nvec; c += G) {
        fetch(c * 8, 0);
        number(0, v[0]);
        if (mine)
          *reinterpret_cast<uint2*>(q + r * ld + c * 8) = i8_round8<MODE>(v[0], k, r * cols + c * 8, k0, k1, role);
      }
    }
  }
}

// 4 x 4 bytes: word i of the result holds byte i of the four words.
__device__ __forceinline__ void transpose4(const uint32_t (&w)[4], uint32_t (&o)[4]) {
  const uint32_t a = __builtin_amdgcn_perm(w[1], w[0], 0x05010400u), b = __builtin_amdgcn_perm(w[3], w[2], 0x05010400u);
  const uint32_t c = __builtin_amdgcn_perm(w[1], w[0], 0x07030602u), d = __builtin_amdgcn_perm(w[3], w[2], 0x07030602u);
  o[0] = __builtin_amdgcn_perm(b, a, 0x05040100u);
  o[1] = __builtin_amdgcn_perm(b, a, 0x07060302u);
  o[2] = __builtin_amdgcn_perm(d, c, 0x05040100u);
  o[3] = __builtin_amdgcn_perm(d, c, 0x07060302u);
}

// The transposed tile in LDS: COLS columns of 32 words (128 tokens), written out as
// rows of 128 bytes.  33 words a column keep both directions off shared banks.
template <int COLS>
using TileT = uint32_t[COLS][33];
template <int COLS>
__device__ __forceinline__ void store_tile_t(const TileT<COLS>& tile, int8_t* qt, int64_t cols, int64_t ldt,
                                             int64_t r0, int64_t c0) {
#pragma unroll
  for (int i = 0; i < COLS / 32; ++i) {
    const int c = (threadIdx.x >> 3) + i * 32, w = (threadIdx.x & 7) * 4;
    if (c0 + c < cols)
      *reinterpret_cast<uint4*>(qt + (c0 + c) * ldt + r0 + w * 4) =
          make_uint4(tile[c][w], tile[c][w + 1], tile[c][w + 2], tile[c][w + 3]);
  }
}

// INT8 [rows][ld] -> [cols][ldt], zeros for the rows past the last.  128 x 128 tiles.
// 8192 x 2048: 6.9 us (4.9 TB/s).
__global__ __launch_bounds__(kBlock) void k_transpose_i8(const int8_t* __restrict__ q, int64_t rows, int64_t cols,
                                                         int64_t ld, int8_t* __restrict__ qt, int64_t ldt,
                                                         uint32_t ctiles) {
  __shared__ TileT<128> tile;
  const int64_t r0 = (int64_t)(blockIdx.x / ctiles) * 128, c0 = (int64_t)(blockIdx.x % ctiles) * 128;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int c4 = threadIdx.x & 31, r4 = (threadIdx.x >> 5) + i * 8;
    uint32_t w[4], o[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int64_t r = r0 + r4 * 4 + j;
      w[j] = r < rows ? *reinterpret_cast<const uint32_t*>(q + r * ld + c0 + c4 * 4) : 0u;
    }
    transpose4(w, o);
#pragma unroll
    for (int j = 0; j < 4; ++j) tile[c4 * 4 + j][r4] = o[j];
  }
  __syncthreads();
  store_tile_t<128>(tile, qt, cols, ldt, r0, c0);
}

// Column maxima of |x[r][c] roww[r]| and column sums of x over slices of the rows:
// workgroups of 64 columns by one slice, 32 rows at a time.  8192 x 2048 BF16: 8.9 us
// (3.8 TB/s; four rows a thread in flight).
template <int T>
__global__ __launch_bounds__(kBlock) void k_col_max(const typename Elem<T>::type* __restrict__ src, int64_t rows,
                                                    int64_t cols, const float* __restrict__ roww, int64_t slice,
                                                    uint32_t cblocks, uint32_t* __restrict__ pmax,
                                                    float* __restrict__ psum) {
  __shared__ __align__(16) uint32_t smax[kBlock / 64][64];
  __shared__ __align__(16) float ssum[kBlock / 64][64];
  const int cv = threadIdx.x & 7, rg = threadIdx.x >> 3;
  const int64_t c0 = (int64_t)(blockIdx.x % cblocks) * 64, c = c0 + cv * 8, part = blockIdx.x / cblocks;
  const int64_t r1 = min(rows, (part + 1) * slice);
  uint32_t mx[8] = {};
  float sum[8] = {};
  constexpr int U = 4;  // rows in flight
  for (int64_t r = part * slice + rg; r < r1; r += 32 * U) {
    Raw<T, 8> raw[U];
    float w[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool in = r + u * 32 < r1;
      w[u] = in ? roww[r + u * 32] : 0.f;
      fetch_n<T, 8>(src + (r + u * 32) * cols + c, in ? cols - c : 0, raw[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float v[8];
      up_n<T, 8>(raw[u], v);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        mx[i] = max(mx[i], __float_as_uint(v[i] * w[u]) & 0x7fffffffu);
        sum[i] += v[i];
      }
    }
  }
  // over the wave's eight rows, then over the waves
#pragma unroll
  for (int o = 8; o < 64; o <<= 1)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      mx[i] = max(mx[i], (uint32_t)__shfl_xor((int)mx[i], o, 64));
      sum[i] += __shfl_xor(sum[i], o, 64);
    }
  if ((threadIdx.x & 63) < 8) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      smax[threadIdx.x >> 6][cv * 8 + i] = mx[i];
      ssum[threadIdx.x >> 6][cv * 8 + i] = sum[i];
    }
  }
  __syncthreads();
  const int t = threadIdx.x;
  if (t < 64 && c0 + t < cols) {
    pmax[part * cols + c0 + t] = max(max(smax[0][t], smax[1][t]), max(smax[2][t], smax[3][t]));
    psum[part * cols + c0 + t] = (ssum[0][t] + ssum[1][t]) + (ssum[2][t] + ssum[3][t]);
  }
}

// x[r][c] roww[r] rounded by column scale into qt [cols][ldt]: tiles of 128 rows x
// 64 columns, a thread 4 x 8 of them.  The columns' scales come from the slices'
// maxima, at most kMostParts of them, in every tile; the first row of tiles writes them
// and the columns' sums (a launch of its own for that took 3.4 to 4.6 us).  8192 x
// 2048 BF16: 10.6 us (4.7 TB/s).
constexpr int kMostParts = 32;
template <int T, int MODE>
__global__ __launch_bounds__(kBlock) void k_col_i8_t(const typename Elem<T>::type* __restrict__ src, int64_t rows,
                                                     int64_t cols, const float* __restrict__ roww,
                                                     const uint32_t* __restrict__ pmax,
                                                     const float* __restrict__ psum, int32_t parts,
                                                     float* __restrict__ scale, float* __restrict__ sums,
                                                     int8_t* __restrict__ qt, int64_t ldt, uint32_t ctiles,
                                                     uint32_t k0, uint32_t k1, uint32_t role) {
  __shared__ TileT<64> tile;
  __shared__ __align__(16) float ks[64], ki[64];
  __shared__ uint32_t wm[kBlock / 64][64];
  __shared__ float wsum[kBlock / 64][64];
  const int64_t r0 = (int64_t)(blockIdx.x / ctiles) * 128, c0 = (int64_t)(blockIdx.x % ctiles) * 64;
  const int c8 = threadIdx.x & 7, r4 = threadIdx.x >> 3;
  const int64_t c = c0 + c8 * 8;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t at = min(c0 + lane, cols - 1);
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < kMostParts / (kBlock / 64); ++i)
    m = max(m, pmax[(int64_t)min(wave + i * (kBlock / 64), parts - 1) * cols + at]);
  wm[wave][lane] = m;
  const bool first = r0 == 0 && sums;
  if (first) {
    float p[kMostParts / (kBlock / 64)], s = 0.f;
#pragma unroll
    for (int i = 0; i < kMostParts / (kBlock / 64); ++i)
      p[i] = psum[(int64_t)min(wave + i * (kBlock / 64), parts - 1) * cols + at];
#pragma unroll
    for (int i = 0; i < kMostParts / (kBlock / 64); ++i) s += wave + i * (kBlock / 64) < parts ? p[i] : 0.f;
    wsum[wave][lane] = s;
  }
  Raw<T, 8> raw[4];
  float v[4][8], weight[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int64_t r = r0 + r4 * 4 + j;
    weight[j] = r < rows ? roww[r] : 0.f;
    fetch_n<T, 8>(src + r * cols + c, r < rows ? cols - c : 0, raw[j]);
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    up_n<T, 8>(raw[j], v[j]);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[j][i] *= weight[j];
  }
  __syncthreads();
  if (wave == 0) {
    const I8Scale s = i8_scale(max(max(wm[0][lane], wm[1][lane]), max(wm[2][lane], wm[3][lane])));
    ks[lane] = s.s;
    ki[lane] = s.inv;
    if (r0 == 0 && c0 + lane < cols) scale[c0 + lane] = s.s;
  } else if (wave == 1 && first && c0 + lane < cols) {
    sums[at] = (wsum[0][lane] + wsum[1][lane]) + (wsum[2][lane] + wsum[3][lane]);
  }
  __syncthreads();
  I8Scale k[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) k[i] = i8_scale_of(ks[c8 * 8 + i], ki[c8 * 8 + i]);
  uint32_t q[4][8];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (MODE == DFP_ROUND_NEAREST && i8_nearest8<true>(v[j], k, q[j])) continue;
    uint32_t u[8] = {};
    if (MODE == DFP_ROUND_STOCHASTIC) words<8>((r0 + r4 * 4 + j) * cols + c, k0, k1, role, u);
#pragma unroll
    for (int i = 0; i < 8; ++i) q[j][i] = (uint32_t)i8_round<MODE>(v[j][i], k[i], u[i]);
  }
  // (a row past the last is a row of zeros: its words are never above F = 0)
#pragma unroll
  for (int i = 0; i < 8; ++i)
    tile[c8 * 8 + i][r4] = k[i].live ? low_bytes(q[0][i], q[1][i], q[2][i], q[3][i]) : 0u;
  __syncthreads();
  store_tile_t<64>(tile, qt, cols, ldt, r0, c0);
}

constexpr int64_t kMaxBlocks = 1 << 22;  // of a grid-stride launch

}  // namespace

dfp_status launch_rows_i8(int32_t type, int32_t rounding, uint64_t seed, uint32_t role, const void* src, int64_t rows,
                          int64_t cols, const float* colw, int8_t* q, float* scale, hipStream_t st) {
  const int64_t ld = i8_ld(cols), nvec = ld / 8;
  const uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
  return with_type(type, [&](auto tc) -> dfp_status {
    constexpr int T = decltype(tc)::value;
    return with_mode(rounding, [&](auto mc) -> dfp_status {
      constexpr int MODE = decltype(mc)::value;
      auto go = [&](auto g, auto nv, auto weighted) -> dfp_status {
        constexpr int G = decltype(g)::value;
        const int64_t blocks = std::min<int64_t>((rows + kBlock / G - 1) / (kBlock / G), kMaxBlocks);
        DFP_LAUNCH(K_I8_ROWS, (k_rows_i8<T, MODE, G, decltype(nv)::value, decltype(weighted)::value>),
                   dim3((unsigned)blocks), dim3(kBlock), 0, st, (const typename Elem<T>::type*)src, rows, cols, ld,
                   colw, q, scale, k0, k1, role);
        return DFP_OK;
      };
      auto by_len = [&](auto weighted) -> dfp_status {
        typedef std::integral_constant<int, 64> Wave;
        typedef std::integral_constant<int, 256> Group;
        // a wave a row up to 2048 (8192 x 2048 BF16 3% faster than by workgroups, timed in turn); by
        // workgroups for few such rows (their waves share the loads) and up to 16384
        if (nvec <= 64) return go(Wave(), std::integral_constant<int, 1>(), weighted);
        if (nvec <= 128) return go(Wave(), std::integral_constant<int, 2>(), weighted);
        if (nvec <= 256 && rows > 512) return go(Wave(), std::integral_constant<int, 4>(), weighted);
        if (nvec <= 256) return go(Group(), std::integral_constant<int, 1>(), weighted);
        if (nvec <= 512) return go(Group(), std::integral_constant<int, 2>(), weighted);
        if (nvec <= 1024) return go(Group(), std::integral_constant<int, 4>(), weighted);
        if (nvec <= 2048) return go(Group(), std::integral_constant<int, 8>(), weighted);
        return go(Group(), std::integral_constant<int, 0>(), weighted);
      };
      return colw ? by_len(std::true_type()) : by_len(std::false_type());
    });
  });
}

dfp_status launch_transpose_i8(const int8_t* q, int64_t rows, int64_t cols, int8_t* qt, hipStream_t st) {
  const int64_t rt = (rows + 127) / 128, ct = (cols + 127) / 128;
  DFP_LAUNCH(K_I8_TRANSPOSE, k_transpose_i8, dim3((unsigned)(rt * ct)), dim3(kBlock), 0, st, q, rows, cols, i8_ld(cols),
             qt, i8_ld(rows), (uint32_t)ct);
  return DFP_OK;
}

ColPlan plan_cols_i8(int64_t rows, int64_t cols) {
  ColPlan p;
  const int64_t cb = (cols + 63) / 64;
  // enough slices for four workgroups a CU, of at least 32 rows
  const int64_t parts =
      std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>((rows + 31) / 32, kMostParts), 1024 / cb));
  p.slice = (rows + parts - 1) / parts;
  p.parts = (rows + p.slice - 1) / p.slice;
  p.bytes = p.parts * 2 * cols * 4;
  return p;
}

dfp_status launch_cols_i8_t(int32_t type, int32_t rounding, uint64_t seed, uint32_t role, const void* src,
                            int64_t rows, int64_t cols, const float* roww, int8_t* qt, float* scale, float* sums,
                            void* ws, hipStream_t st) {
  const ColPlan p = plan_cols_i8(rows, cols);
  uint32_t* pmax = (uint32_t*)ws;
  float* psum = (float*)(pmax + p.parts * cols);
  const uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
  const int64_t rt = (rows + 127) / 128, ct = (cols + 63) / 64;
  return with_type(type, [&](auto tc) -> dfp_status {
    constexpr int T = decltype(tc)::value;
    typedef const typename Elem<T>::type* S;
    DFP_LAUNCH(K_I8_COLS, k_col_max<T>, dim3((unsigned)(ct * p.parts)), dim3(kBlock), 0, st, (S)src, rows, cols, roww,
               p.slice, (uint32_t)ct, pmax, psum);
    return with_mode(rounding, [&](auto mc) -> dfp_status {
      DFP_LAUNCH(K_I8_COLS, (k_col_i8_t<T, decltype(mc)::value>), dim3((unsigned)(rt * ct)), dim3(kBlock), 0, st,
                 (S)src, rows, cols, roww, pmax, psum, (int32_t)p.parts, scale, sums, qt, i8_ld(rows),
                 (uint32_t)ct, k0, k1, role);
      return DFP_OK;
    });
  });
}

}  // namespace dfp
