// The tiled matrix product shared by the INT8 linear layers and the
// orthogonalised update: D[i][j] = sum over t of A[i][t] B[j][t], both operands
// with the reduction contiguous, in rows of whole 128-byte pieces.  A piece is
//   I8     128 integers                       one product in INT32
//   F16    64 f16 numbers                     one product in FP32
//   F16X2  32 numbers as 32 f16 high parts, then 32 f16 low parts
//          x = hi + lo: hi hi' + hi lo' + lo hi' in FP32 (lo lo' is below 2^-22
//          of the product and left out)
// In all three an MFMA operand register quad is 16 consecutive bytes of a row,
// lanes l and l + 16 k holding row l's quads k = 0 .. 3 (64 bytes), so that one
// loop over pieces serves them.
#pragma once

#include "dfp_internal.h"

namespace dfp {

enum class Prod { I8, F16, F16X2 };

typedef int mv4i __attribute__((ext_vector_type(4)));
typedef float mv4f __attribute__((ext_vector_type(4)));
typedef _Float16 mv8h __attribute__((ext_vector_type(8)));

template <Prod P>
struct MmaTypes {
  typedef mv4f acc_t;
};
template <>
struct MmaTypes<Prod::I8> {
  typedef mv4i acc_t;
};

template <Prod P>
__device__ __forceinline__ typename MmaTypes<P>::acc_t mma16(const mv4i& rows, const mv4i& cols,
                                                             const typename MmaTypes<P>::acc_t& c) {
  if constexpr (P == Prod::I8)
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(rows, cols, c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(mv8h, rows), __builtin_bit_cast(mv8h, cols), c, 0,
                                                  0, 0);
}

constexpr int kPiece = 128;  // bytes of a row per step of the loop

// One workgroup's TM x TN tile by WM x WN waves.  Lane l of wave (wm, wn) ends
// with acc[i][j][r] = D[wm TM/WM + 16 i + l % 16][wn TN/WN + 16 j + 4 (l / 16) + r]:
// four consecutive columns of one row (the B rows are the MFMA's first operand).
template <Prod P, int TM, int TN, int WM, int WN>
struct MmaTile {
  typedef typename MmaTypes<P>::acc_t acc_t;
  static constexpr int kThreads = 64 * WM * WN;
  static constexpr int FM = TM / WM / 16, FN = TN / WN / 16;
  static constexpr int kLoadsA = TM * 8 / kThreads, kLoadsB = TN * 8 / kThreads;  // 16-byte pieces of a thread
  static constexpr int kStage = (TM + TN) * kPiece;
  static constexpr int kLds = 2 * kStage;
  static_assert(TM * 8 % kThreads == 0 && TN * 8 % kThreads == 0, "whole loads");

  // a, b: the tile's first rows; rows past na, nb (counted from there) repeat the
  // last one, what comes of them is for the caller to drop.  pieces >= 1.
  // Two LDS stages: while the MFMAs run on one, the next step's rows are on their
  // way into registers; they are stored once this step's reads are done.  A row's
  // 16-byte quads are permuted by (quad ^ row % 8), which spreads the 16 rows that
  // an operand read takes over all banks.
  static __device__ __forceinline__ void run(const uint8_t* __restrict__ a, int64_t lda, int32_t na,
                                             const uint8_t* __restrict__ b, int64_t ldb, int32_t nb, int32_t pieces,
                                             uint8_t* smem, acc_t (&acc)[FM][FN]) {
    const int t = threadIdx.x;
    const int lane = t & 63, wave = t >> 6;
    const int wm = wave / WN, wn = wave % WN;
    uint32_t offa[kLoadsA], offb[kLoadsB];
#pragma unroll
    for (int i = 0; i < kLoadsA; ++i)
      offa[i] = (uint32_t)(min((t >> 3) + i * (kThreads / 8), na - 1) * lda) + (t & 7) * 16;
#pragma unroll
    for (int i = 0; i < kLoadsB; ++i)
      offb[i] = (uint32_t)(min((t >> 3) + i * (kThreads / 8), nb - 1) * ldb) + (t & 7) * 16;
    // (kThreads / 8 is a multiple of 8: a thread's rows have one permutation)
    const uint32_t st = (t >> 3) * kPiece + (((t & 7) ^ ((t >> 3) & 7)) << 4);
    const int r = lane & 15, g = lane >> 4;
    const uint32_t fa = (wm * (TM / WM) + r) * kPiece + ((g ^ (r & 7)) << 4);
    const uint32_t fb = TM * kPiece + (wn * (TN / WN) + r) * kPiece + ((g ^ (r & 7)) << 4);

    mv4i ra[kLoadsA], rb[kLoadsB];
    auto fetch = [&](int32_t p) {
      const uint8_t* pa = a + (int64_t)p * kPiece;
      const uint8_t* pb = b + (int64_t)p * kPiece;
#pragma unroll
      for (int i = 0; i < kLoadsA; ++i) ra[i] = *(const mv4i*)(pa + offa[i]);
#pragma unroll
      for (int i = 0; i < kLoadsB; ++i) rb[i] = *(const mv4i*)(pb + offb[i]);
    };
    auto store = [&](uint32_t stage) {
      uint8_t* d = smem + stage + st;
#pragma unroll
      for (int i = 0; i < kLoadsA; ++i) *(mv4i*)(d + i * (kThreads / 8) * kPiece) = ra[i];
#pragma unroll
      for (int i = 0; i < kLoadsB; ++i) *(mv4i*)(d + TM * kPiece + i * (kThreads / 8) * kPiece) = rb[i];
    };

#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) acc[i][j] = acc_t{0, 0, 0, 0};

    fetch(0);
    store(0);
    if (pieces > 1) fetch(1);
    __syncthreads();
    for (int32_t p = 0; p < pieces; ++p) {
      const uint32_t stage = (p & 1) * kStage;
      const uint8_t* sa = smem + stage + fa;
      const uint8_t* sb = smem + stage + fb;
      mv4i qa[2][FM], qb[2][FN];
      // quads g and 4 + g of every row: the second is the first with bit 6 turned
      auto read_a = [&](int h) {
#pragma unroll
        for (int i = 0; i < FM; ++i)
          qa[h][i] = *(const mv4i*)(smem + (((uint32_t)(sa - smem)) ^ (h * 64)) + i * 16 * kPiece);
      };
      auto read_b = [&](int h) {
#pragma unroll
        for (int j = 0; j < FN; ++j)
          qb[h][j] = *(const mv4i*)(smem + (((uint32_t)(sb - smem)) ^ (h * 64)) + j * 16 * kPiece);
      };
      auto product = [&](int ha, int hb) {
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
          for (int j = 0; j < FN; ++j) acc[i][j] = mma16<P>(qb[hb][j], qa[ha][i], acc[i][j]);
      };
      read_a(0);
      read_b(0);
      if constexpr (P == Prod::F16X2) {
        read_b(1);
        product(0, 0);
        product(0, 1);
        read_a(1);
        product(1, 0);
      } else {
        product(0, 0);
        read_a(1);
        read_b(1);
        product(1, 1);
      }
      if (p + 1 < pieces) {
        store(kStage - stage);
        if (p + 2 < pieces) fetch(p + 2);
      }
      __syncthreads();
    }
  }
};

// Workgroup -> tile: consecutive workgroups go round the 8 XCDs, each with an L2
// of its own.  An XCD takes a contiguous run of tiles, walked in bands of `band`
// tile rows, so that the tiles it has in flight share rows of both operands.
__device__ __forceinline__ void tile_of(uint32_t id, uint32_t tm, uint32_t tn, uint32_t band, uint32_t* im,
                                        uint32_t* in) {
  const uint32_t total = tm * tn, xcd = id & 7, q = total >> 3, rem = total & 7;
  const uint32_t t = xcd * q + min(xcd, rem) + (id >> 3);
  const uint32_t per = band * tn, b = t / per, first = b * band, h = min(band, tm - first), w = t - b * per;
  *im = first + w % h;
  *in = w / h;
}

}  // namespace dfp
