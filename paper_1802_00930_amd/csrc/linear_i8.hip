// INT8 products with a scale per row of either operand: out[i][j] =
// (sum over t of a[i][t] b[j][t]) sa[i] sb[j] + bias[j], the sum exact in INT32,
// so that it may be cut anywhere and added in any order with the same result.
//   k_few    few rows (one token, a decoding batch): bound by the weights' bytes
//   k_tiles  tiles of outputs on the loop of mma_tile.h, the reduction cut into
//            slices where the tiles alone leave CUs idle; k_slices adds those up
#include <type_traits>

#include "dfp_internal.h"
#include "dfp_types.h"
#include "i8_round.h"
#include "linear_i8.h"
#include "mma_tile.h"

#pragma clang fp contract(off)

namespace dfp {

namespace {

struct I8Args {
  const uint8_t *a, *b;
  const float *sa, *sb, *bias;  // sb, bias nullable
  void* out;
  int32_t* part;  // slices: [slice][m][n]
  int64_t ld;     // bytes of an operand row
  int32_t m, n;
  uint32_t tm, tn;
  int32_t per;    // pieces of a slice
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

// SLICED: the tiles of every slice in turn, their sums to g.part.
// 16384 x 8192 x 8192 BF16 out: 855 to 1002 us (2570 to 2190 TOP/s, by card and how hot it
// runs); 4096^3 61 us (2240 TOP/s: one round of tiles that start and end together).
template <int T, bool SLICED, class Q>
__global__ __launch_bounds__(Q::kThreads, 2) void k_tiles(I8Args g) {
  typedef typename Q::template Tile<Prod::I8> Tile;
  constexpr int TM = Q::TM, TN = Q::TN, WM = Q::WM, WN = Q::WN;
  const uint32_t id = xcd_order(blockIdx.x, gridDim.x), tiles = g.tm * g.tn, slice = SLICED ? id / tiles : 0;
  uint32_t im, in;
  tile_of(id - slice * tiles, g.tm, g.tn, 8, &im, &in);
  const int64_t i0 = (int64_t)im * TM, j0 = (int64_t)in * TN;
  const int32_t p0 = (int32_t)slice * g.per;
  const int32_t pieces = SLICED ? min(g.per, (int32_t)(g.ld / kPiece) - p0) : (int32_t)(g.ld / kPiece);
  // The tile's scales wait in LDS: loaded where they are used, after the product,
  // they cost 2 us of memory's latency (1500 x 2048 x 128: 6.1 us in all).
  __shared__ __align__(16) float fa[TM], fb[TN], fbias[TN];
  if (!SLICED) {
    for (int t = threadIdx.x; t < TM; t += Q::kThreads) fa[t] = g.sa[min(i0 + t, (int64_t)g.m - 1)];
    for (int t = threadIdx.x; t < TN; t += Q::kThreads) {
      const int64_t c = min(j0 + t, (int64_t)g.n - 1);
      fb[t] = g.sb ? g.sb[c] : 1.f;
      fbias[t] = g.bias ? g.bias[c] : 0.f;
    }
  }
  mv4i acc[Tile::FM][Tile::FN];
  Tile::run(g.a + i0 * g.ld + (int64_t)p0 * kPiece, g.ld, (int32_t)(g.m - i0),
            g.b + j0 * g.ld + (int64_t)p0 * kPiece, g.ld, (int32_t)(g.n - j0), pieces, acc);
  if (threadIdx.x >= Tile::kThreads) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t i1 = i0 + (wave / WN) * (TM / WM) + (lane & 15);
  const int64_t j1 = j0 + (wave % WN) * (TN / WN) + (lane >> 4) * 8;
  // 64 or 96 columns of a row one after the other: of 16-bit outputs a store is half a
  // line, and a tile's lines leave L2 before a half that comes later joins them
  constexpr int JN = Tile::FN % 4 == 0 ? 4 : Tile::FN % 6 == 0 ? 6 : 2;
#pragma unroll
  for (int j = 0; j < Tile::FN; j += JN) {
    float sb[JN / 2][8], bias[JN / 2][8];
    if (!SLICED) {
#pragma unroll
      for (int h = 0; h < JN / 2; ++h)
#pragma unroll
        for (int r = 0; r < 8; ++r) {
          const int64_t c = j1 - j0 + (j + 2 * h) * 16 + r;
          sb[h][r] = fb[c], bias[h][r] = fbias[c];
        }
    }
#pragma unroll
    for (int i = 0; i < Tile::FM; ++i) {
      const int64_t ii = i1 + i * 16;
      if (ii >= g.m) continue;
#pragma unroll
      for (int h = 0; h < JN / 2; ++h) {
        const int64_t jj = j1 + (j + 2 * h) * 16;
        if (jj >= g.n) continue;
        float v[8];
#pragma unroll
        for (int r = 0; r < 8; ++r) {
          const int32_t s = acc[i][j + 2 * h + (r >> 2)][r & 3];
          if (SLICED) {
            v[r] = __int_as_float(s);  // stored as it is
          } else {
            v[r] = (float)s * fa[ii - i0] * sb[h][r];
            if (g.bias) v[r] = v[r] + bias[h][r];
          }
        }
        if (SLICED)
          store_n<DFP_F32, 8>((float*)g.part + ((int64_t)slice * g.m + ii) * g.n + jj, g.n - jj, v);
        else
          store_n<T, 8>((typename Elem<T>::type*)g.out + ii * g.n + jj, g.n - jj, v);
      }
    }
  }
}

// The slices' sums, four columns of a row a thread: bound by the launch and a trip to
// memory (4 us), then by the sums' bytes.
template <int T>
__global__ __launch_bounds__(256) void k_slices(I8Args g, int32_t slices) {
  const int64_t nq = (g.n + 3) / 4, id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t i = id / nq, j = id % nq * 4;
  if (i >= g.m) return;
  mv4i s = {0, 0, 0, 0};
  const float* p = (const float*)g.part + i * g.n + j;
  for (int32_t k = 0; k < slices; k += 8) {  // eight loads in flight
    float v[8][4];
#pragma unroll
    for (int u = 0; u < 8; ++u)
      load_n<DFP_F32, 4>(p + (int64_t)min(k + u, slices - 1) * g.m * g.n, g.n - j, v[u]);
#pragma unroll
    for (int u = 0; u < 8; ++u)
#pragma unroll
      for (int r = 0; r < 4; ++r) s[r] += k + u < slices ? __float_as_int(v[u][r]) : 0;
  }
  store_quad<T>(g, i, j, s);
}

// Few rows.  A workgroup takes 16 columns of up to 16 RT rows over the whole
// reduction: its waves deal out the pieces among them, every lane reading 16 bytes
// of a weight row straight into an MFMA operand (no LDS: nothing is read twice),
// and their sums meet in LDS.  Bound by the latency of the weights' bytes: 16 rows by
// 4096 x 4096 7.9 us (2.1 TB/s), by 8192 x 8192 19.4 us (3.5 TB/s).
constexpr int kFewWaves = 8;
constexpr int kTokenRows = 2;
constexpr int kTokenVecs = 8;                                        // of 8 elements, a lane's share of a row
constexpr int kTokenBytes = 64 * 8 * kTokenVecs * kFewWaves + 16 * kTokenRows;  // all waves' rows, and their padding
// log2 of the waves that share a row of x
__host__ __device__ __forceinline__ int32_t token_shift(int64_t m) { return m == 1 ? 3 : 2; }
template <int T, int RT, int UNROLL>
__global__ __launch_bounds__(64 * kFewWaves) void k_few(I8Args g) {
  __shared__ int32_t part[kFewWaves][RT * 256];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t j0 = (int64_t)blockIdx.x * 16;
  const int32_t pieces = (int32_t)(g.ld / kPiece);
  const uint8_t* pb = g.b + min(j0 + (lane & 15), (int64_t)g.n - 1) * g.ld + (lane >> 4) * 16;
  const uint8_t* pa[RT];
#pragma unroll
  for (int i = 0; i < RT; ++i) pa[i] = g.a + (int64_t)min((lane & 15) + i * 16, g.m - 1) * g.ld + (lane >> 4) * 16;
  mv4i acc[RT];
#pragma unroll
  for (int i = 0; i < RT; ++i) acc[i] = mv4i{0, 0, 0, 0};
  for (int32_t p = wave; p < pieces; p += kFewWaves * UNROLL) {
    mv4i b[UNROLL][2], a[UNROLL][RT][2];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      const int64_t at = (int64_t)min(p + u * kFewWaves, pieces - 1) * kPiece;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        b[u][h] = *(const mv4i*)(pb + at + h * 64);
#pragma unroll
        for (int i = 0; i < RT; ++i) a[u][i][h] = *(const mv4i*)(pa[i] + at + h * 64);
      }
    }
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      if (p + u * kFewWaves >= pieces) break;
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < RT; ++i) acc[i] = mma16<Prod::I8>(b[u][h], a[u][i][h], acc[i]);
    }
  }
#pragma unroll
  for (int i = 0; i < RT; ++i) *(mv4i*)&part[wave][i * 256 + lane * 4] = acc[i];
  __syncthreads();
  for (int q = threadIdx.x; q < RT * 64; q += 64 * kFewWaves) {
    mv4i s = {0, 0, 0, 0};
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) s += *(const mv4i*)&part[w][q * 4];
    const int64_t i = (q >> 6) * 16 + (q & 15), j = j0 + ((q >> 4) & 3) * 4;
    if (i < g.m && j < g.n) store_quad<T>(g, i, j, s);
  }
}

// One token or a few, quantised on the way: every workgroup of k_few's kind turns
// the rows of x into INT8 in its own LDS, which takes the launch of a quantiser out
// of the call.  The first pieces of the weights are on their way meanwhile, requested
// after the row, since loads are waited for in order (one row by 4096 x 4096 7.4 us, 2.3
// TB/s; before the row 8.4, in two launches 10.9).  The row stays packed, in 128 registers
// with all else, so that two workgroups share a CU (one row by 8192 x 8192: 16.2 us,
// with one 19.3).  Stochastic rounding does not fit them, its row spills (144 to 272 bytes a
// lane; one row by 4096 x 4096 13.4 us a call, nearest 6.8).
template <int T, int MODE, int UNROLL>
__global__ __launch_bounds__(64 * kFewWaves, 4) void k_token(I8Args g, const typename Elem<T>::type* __restrict__ x,
                                                          int32_t k, uint32_t k0, uint32_t k1) {
  __shared__ __align__(16) uint8_t xq[kTokenBytes];
  __shared__ int32_t part[kFewWaves][256];
  __shared__ uint32_t red[kFewWaves];
  __shared__ float sx[kTokenRows];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t j0 = (int64_t)blockIdx.x * 16;
  const int32_t pieces = (int32_t)(g.ld / kPiece), stride = (int32_t)g.ld + 16;  // 16: rows on other banks
  const uint8_t* pb = g.b + min(j0 + (lane & 15), (int64_t)g.n - 1) * g.ld + (lane >> 4) * 16;
  mv4i b[UNROLL][2];
  auto fetch = [&](int32_t p) {
#pragma unroll
    for (int u = 0; u < UNROLL; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h)
        b[u][h] = *(const mv4i*)(pb + (int64_t)min(p + u * kFewWaves, pieces - 1) * kPiece + h * 64);
  };
  // eight or four waves a row; the row stays in registers
  const int32_t sh = token_shift(g.m), row = wave >> sh, sub = wave & ((1 << sh) - 1);
  Raw<T, 8> raw[kTokenVecs];
  uint32_t mx = 0;
#pragma unroll
  for (int i = 0; i < kTokenVecs; ++i) {
    const int32_t c = ((i << sh | sub) * 64 + lane) * 8;
    fetch_n<T, 8>(x + (int64_t)row * k + c, row < g.m ? k - c : 0, raw[i]);
  }
  fetch(wave);
#pragma unroll
  for (int i = 0; i < kTokenVecs; ++i) {
    float v[8];
    up_n<T, 8>(raw[i], v);
#pragma unroll
    for (int e = 0; e < 8; ++e) mx = max(mx, __float_as_uint(v[e]) & 0x7fffffffu);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) mx = max(mx, (uint32_t)__shfl_xor((int)mx, o, 64));
  if (lane == 0) red[wave] = mx;
  __syncthreads();
  for (int w = 0; w < 1 << sh; ++w) mx = max(mx, red[(row << sh) + w]);
  const I8Scale sc = i8_scale(mx);
  if (sub == 0 && lane == 0) sx[row] = sc.s;
#pragma unroll
  for (int i = 0; i < kTokenVecs; ++i) {
    const int32_t c = ((i << sh | sub) * 64 + lane) * 8;
    float v[8];
    up_n<T, 8>(raw[i], v);
    if (row < g.m && c < (int32_t)g.ld)
      *(uint2*)(xq + row * stride + c) = i8_round8<MODE>(v, sc, (int64_t)row * k + c, k0, k1, DFP_ROLE_X);
  }
  __syncthreads();
  const uint8_t* pa = xq + min(lane & 15, g.m - 1) * stride + (lane >> 4) * 16;
  mv4i acc = {0, 0, 0, 0};
  for (int32_t p = wave; p < pieces; p += kFewWaves * UNROLL) {
    mv4i w[UNROLL][2];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) w[u][0] = b[u][0], w[u][1] = b[u][1];
    if (p + kFewWaves * UNROLL < pieces) fetch(p + kFewWaves * UNROLL);
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      if (p + u * kFewWaves >= pieces) break;
#pragma unroll
      for (int h = 0; h < 2; ++h)
        acc = mma16<Prod::I8>(w[u][h], *(const mv4i*)(pa + (p + u * kFewWaves) * kPiece + h * 64), acc);
    }
  }
  *(mv4i*)&part[wave][lane * 4] = acc;
  __syncthreads();
  if (threadIdx.x < 64) {
    mv4i s = {0, 0, 0, 0};
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) s += *(const mv4i*)&part[w][lane * 4];
    const int64_t i = lane & 15, j = j0 + (lane >> 4) * 4;
    g.sa = sx;
    if (i < g.m && j < g.n) store_quad<T>(g, i, j, s);
  }
}

}  // namespace

bool fits_token_i8(int64_t m, int64_t k) {
  return m <= kTokenRows && i8_ld(k) <= (int64_t)64 * 8 * kTokenVecs << token_shift(m);
}

dfp_status launch_token_i8(int32_t m, int32_t n, int32_t k, int32_t type, int32_t rounding, uint64_t seed,
                           const void* x, const int8_t* b, const float* sb, const float* bias, void* out,
                           hipStream_t st) {
  I8Args g{nullptr, (const uint8_t*)b, nullptr, sb, bias, out, nullptr, i8_ld(k), m, n, 0, 0, 0};
  return with_type(type, [&](auto tc) -> dfp_status {
    constexpr int T = decltype(tc)::value;
    return with_mode(rounding, [&](auto mc) -> dfp_status {
      DFP_LAUNCH(K_I8_GEMM, (k_token<T, decltype(mc)::value, 4>), dim3((unsigned)(((int64_t)n + 15) / 16)),
                 dim3(64 * kFewWaves), 0, st, g, (const typename Elem<T>::type*)x, k, (uint32_t)seed,
                 (uint32_t)(seed >> 32));
      return DFP_OK;
    });
  });
}

dfp_status launch_gemm_i8(int32_t m, int32_t n, int32_t k, const int8_t* a, const float* sa, const int8_t* b,
                          const float* sb, const float* bias, int32_t type, void* out, void* ws, hipStream_t st) {
  const I8Plan p = plan_gemm_i8(m, n, k);
  I8Args g{(const uint8_t*)a, (const uint8_t*)b, sa, sb, bias, out, (int32_t*)ws, i8_ld(k), m, n, 0, 0, p.per};
  return with_type(type, [&](auto tc) -> dfp_status {
    constexpr int T = decltype(tc)::value;
    if (p.kind < 0) {
      const dim3 grid((unsigned)(((int64_t)n + 15) / 16)), block(64 * kFewWaves);
      if (m <= 16)
        DFP_LAUNCH(K_I8_GEMM, (k_few<T, 1, 4>), grid, block, 0, st, g);
      else if (m <= 32)
        DFP_LAUNCH(K_I8_GEMM, (k_few<T, 2, 4>), grid, block, 0, st, g);
      else
        DFP_LAUNCH(K_I8_GEMM, (k_few<T, 4, 4>), grid, block, 0, st, g);
      return DFP_OK;
    }
    g.tm = (uint32_t)(((int64_t)m + kTileKinds[p.kind].tm - 1) / kTileKinds[p.kind].tm);
    g.tn = (uint32_t)(((int64_t)n + kTileKinds[p.kind].tn - 1) / kTileKinds[p.kind].tn);
    auto tiles = [&](auto sliced) -> dfp_status {
      constexpr bool SL = decltype(sliced)::value;
      // (a sliced kernel stores integers: one instance serves every type)
      constexpr int TT = SL ? DFP_F32 : T;
      return with_tile(p.kind, [&](auto shape) -> dfp_status {
        typedef decltype(shape) Q;
        DFP_LAUNCH(K_I8_GEMM, (k_tiles<TT, SL, Q>), dim3(g.tm * g.tn * (unsigned)p.slices), dim3(Q::kThreads), 0, st,
                   g);
        return DFP_OK;
      });
    };
    if (p.slices == 1) return tiles(std::false_type());
    const dfp_status rc = tiles(std::true_type());
    if (rc != DFP_OK) return rc;
    const int64_t quads = (int64_t)m * (((int64_t)n + 3) / 4);
    DFP_LAUNCH(K_I8_GEMM, k_slices<T>, dim3((unsigned)((quads + 255) / 256)), dim3(256), 0, st, g, p.slices);
    return DFP_OK;
  });
}

}  // namespace dfp
