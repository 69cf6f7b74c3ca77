// INT8 products with a scale per row of either operand: out[i][j] =
// (sum over t of a[i][t] b[j][t]) sa[i] sb[j] + bias[j], the sum exact in INT32.
#include <algorithm>
#include <type_traits>

#include "dfp_internal.h"
#include "dfp_types.h"
#include "linear_i8.h"
#include "mma_tile.h"

#pragma clang fp contract(off)

namespace dfp {

namespace {

struct I8Args {
  const uint8_t *a, *b;
  const float *sa, *sb, *bias;  // sb, bias nullable
  void* out;
  int64_t ld;  // bytes of an operand row
  int32_t m, n;
  uint32_t tm, tn;
};

// One output quad: four consecutive columns j of row i.
template <int T>
__device__ __forceinline__ void store_quad(const I8Args& g, int64_t i, int64_t j, const mv4i& s) {
  const float sa = g.sa[i];
  float v[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int64_t c = min(j + r, (int64_t)g.n - 1);
    v[r] = (float)s[r] * sa;
    if (g.sb) v[r] = v[r] * g.sb[c];
    if (g.bias) v[r] = v[r] + g.bias[c];
  }
  store_n<T, 4>((typename Elem<T>::type*)g.out + i * g.n + j, g.n - j, v);
}

template <int T, int TM, int TN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) void k_gemm_i8(I8Args g) {
  typedef MmaTile<Prod::I8, TM, TN, WM, WN> Tile;
  __shared__ __align__(16) uint8_t smem[Tile::kLds];
  uint32_t im, in;
  tile_of(blockIdx.x, g.tm, g.tn, 8, &im, &in);
  const int64_t i0 = (int64_t)im * TM, j0 = (int64_t)in * TN;
  mv4i acc[Tile::FM][Tile::FN];
  Tile::run(g.a + i0 * g.ld, g.ld, (int32_t)(g.m - i0), g.b + j0 * g.ld, g.ld, (int32_t)(g.n - j0),
            (int32_t)(g.ld / kPiece), smem, acc);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t i1 = i0 + (wave / WN) * (TM / WM) + (lane & 15);
  const int64_t j1 = j0 + (wave % WN) * (TN / WN) + (lane >> 4) * 4;
#pragma unroll
  for (int i = 0; i < Tile::FM; ++i)
#pragma unroll
    for (int j = 0; j < Tile::FN; ++j)
      if (i1 + i * 16 < g.m && j1 + j * 16 < g.n) store_quad<T>(g, i1 + i * 16, j1 + j * 16, acc[i][j]);
}

}  // namespace

dfp_status launch_gemm_i8(int32_t m, int32_t n, int32_t k, const int8_t* a, const float* sa, const int8_t* b,
                          const float* sb, const float* bias, int32_t type, void* out, hipStream_t st) {
  I8Args g{(const uint8_t*)a, (const uint8_t*)b, sa, sb, bias, out, i8_ld(k), m, n, 0, 0};
  return with_type(type, [&](auto tc) -> dfp_status {
    constexpr int T = decltype(tc)::value;
    g.tm = (uint32_t)(((int64_t)m + 127) / 128);
    g.tn = (uint32_t)(((int64_t)n + 127) / 128);
    DFP_LAUNCH(K_I8_GEMM, (k_gemm_i8<T, 128, 128, 2, 2>), dim3(g.tm * g.tn), dim3(256), 0, st, g);
    return DFP_OK;
  });
}

}  // namespace dfp
