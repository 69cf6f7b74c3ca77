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

#include <type_traits>
#include <utility>

#include "dfp_internal.h"
#include "mm_plan.h"

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

typedef __attribute__((address_space(3))) void* mma_lds_t;

// One workgroup's TM x TN tile by WM x WN waves.  Lane l of wave (wm, wn) ends
// with acc[i][j][r] = D[wm TM/WM + 16 i + l % 16][wn TN/WN + 32 (j / 2) + 8 (l / 16) +
// 4 (j % 2) + r]: of a pair of j, eight consecutive columns of one row, 16 bytes of
// a 16-bit output (the B rows are the MFMA's first operand, and lane x of a
// fragment reads row 8 (x / 4) + x % 4 of its 32, four further on for odd j).
//
// A ring of S LDS stages: the piece S - 1 ahead goes straight to LDS (16 bytes a
// lane) while the MFMAs run on this one, with one barrier a piece.  The stages
// are arrays of their own, not parts of one, so that the compiler sees that a
// stage's reads do not wait for the loads into the others.  A row's 16-byte quads
// are permuted by an XOR with three bits of the row, at the source address since
// the LDS side of such a load is linear: row bits 0 - 2 for A, 0, 1 and 3 for B,
// which differ in the eight rows that are read at once: no bank conflicts.
// 8192 x 8192 outputs, 8192 bytes a row, 256 x 256 tiles by 4 x 2 waves: I8 480 us,
// 2290 TOP/s (library 2331), F16 486 us, 1130 TFLOP/s (1483), F16X2 600 us, 1380 of its 3
// products, by card 4 % either way.  The MFMAs run 54 and 68 % of the cycles; LDS
// is half idle.  A part of that is the card's power: operands of zeros take 424, 422
// and 480 us.  Left: staging through registers (2240, 1110 and 1210), 128 x 128 outputs a
// wave, one wave a SIMD, the next half's reads between this half's MFMAs (2230, 1100 and
// 1370), two groups of waves that take turns between reads and MFMAs, four barriers a
// piece (I8 2070), 32 x 32 MFMAs and deeper rings (no gain).
//
// KG > 1: as many groups of WM x WN waves take the pieces in turn, each with a ring of
// its own, and group 0 ends with the sums of all: for a CU that has one tile, where a
// group spends much of its time waiting (64 x 64, 512 x 512 x 8192 bytes: 20.6 us, two
// groups 15.9, three 15.5: 28 bytes a clock then come from L2 to the CU).
template <Prod P, int TM, int TN, int WM, int WN, int S, int KG>
struct MmaTile {
  typedef typename MmaTypes<P>::acc_t acc_t;
  static constexpr int kThreads = 64 * WM * WN;  // of a group
  static constexpr int FM = TM / WM / 16, FN = TN / WN / 16;
  static constexpr int kLoadsA = TM * 8 / kThreads, kLoadsB = TN * 8 / kThreads;  // 16-byte quads of a thread
  static constexpr int kStage = (TM + TN) * kPiece;
  static_assert(TM * 8 % kThreads == 0 && TN * 8 % kThreads == 0, "whole loads");
  // (kThreads / 8 rows a load, a multiple of 16: a thread's rows have one permutation)
  static_assert(kThreads % 128 == 0 && FN % 2 == 0, "row bits 0 - 3 of a thread's loads; pairs of j");

  template <class F, int... I>
  static __device__ __forceinline__ void for_each(F f, std::integer_sequence<int, I...>) {
    (f(std::integral_constant<int, I>()), ...);
  }
  template <class F>
  static __device__ __forceinline__ void for_stages(F f) {
    for_each(f, std::make_integer_sequence<int, S>());
  }
  template <int I>
  static __device__ __forceinline__ uint8_t* stage() {
    __shared__ __align__(16) uint8_t s[KG * kStage];
    return s;
  }

  // a, b: the tile's first rows; rows past na, nb (counted from there) repeat the
  // last one, what comes of them is for the caller to drop.  pieces >= 1; a tile's
  // rows span less than 2^31 bytes.
  static __device__ __forceinline__ void run(const uint8_t* a, int64_t lda, int32_t na, const uint8_t* b, int64_t ldb,
                                             int32_t nb, int32_t pieces, acc_t (&acc)[FM][FN]) {
    const int kg = KG > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / kThreads) : 0;
    const int t = threadIdx.x - kg * kThreads;
    const int lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int wm = wave / WN, wn = wave % WN;
    int32_t offa[kLoadsA], offb[kLoadsB];
    const int row = t >> 3;
    const int32_t qa16 = ((t & 7) ^ (row & 7)) * 16, qb16 = ((t & 7) ^ ((row & 3) | ((row >> 1) & 4))) * 16;
#pragma unroll
    for (int i = 0; i < kLoadsA; ++i) offa[i] = (int32_t)(min(row + i * (kThreads / 8), na - 1) * lda) + qa16;
#pragma unroll
    for (int i = 0; i < kLoadsB; ++i) offb[i] = (int32_t)(min(row + i * (kThreads / 8), nb - 1) * ldb) + qb16;
    const __amdgpu_buffer_rsrc_t ra =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(a), (short)0, 0x7fffffff, 0x00020000);
    const __amdgpu_buffer_rsrc_t rb =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(b), (short)0, 0x7fffffff, 0x00020000);
    const int r = lane & 15, g = lane >> 4;
    const uint32_t fa = (wm * (TM / WM) + r) * kPiece + ((g ^ (r & 7)) << 4);
    // B: row 8 (r / 4) + r % 4, whose permutation bits are r's own 0 - 2
    const uint32_t fb = TM * kPiece + (wn * (TN / WN) + (r >> 2) * 8 + (r & 3)) * kPiece + ((g ^ (r & 7)) << 4);
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) acc[i][j] = acc_t{0, 0, 0, 0};

    // (step q: piece q KG + kg)
    auto fetch = [&](int32_t q, uint8_t* base) {
      uint8_t* s = base + kg * kStage;
      const int32_t p = min(q * KG + kg, pieces - 1);
#pragma unroll
      for (int i = 0; i < kLoadsA; ++i)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (mma_lds_t)(s + (i * kThreads + wave * 64) * 16), 16, offa[i],
                                                 p * kPiece, 0, 0);
#pragma unroll
      for (int i = 0; i < kLoadsB; ++i)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, (mma_lds_t)(s + TM * kPiece + (i * kThreads + wave * 64) * 16),
                                                 16, offb[i], p * kPiece, 0, 0);
      __builtin_amdgcn_sched_barrier(0);  // not behind the reads of the other stage
    };
    auto compute = [&](const uint8_t* base) {
      const uint8_t* s = base + kg * kStage;
      mv4i qa[2][FM], qb[2][FN];
      // quads g and 4 + g of every row: the second is the first with bit 6 turned
      auto read_a = [&](int h) {
#pragma unroll
        for (int i = 0; i < FM; ++i) qa[h][i] = *(const mv4i*)(s + (fa ^ (h * 64)) + i * 16 * kPiece);
      };
      auto read_b = [&](int h) {
#pragma unroll
        for (int j = 0; j < FN; ++j) qb[h][j] = *(const mv4i*)(s + (fb ^ (h * 64)) + ((j >> 1) * 32 + (j & 1) * 4) * kPiece);
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
    };

    // Past the last piece the loads repeat it, into stages that nothing reads any
    // more: the number in flight stays the same.
    auto step = [&](int32_t q, auto at) {
      constexpr int I = decltype(at)::value;
      __builtin_amdgcn_sched_barrier(0);
      // This wave's loads of piece q have landed, then everybody's, and everybody is
      // done reading q - 1.  (As assembly: the compiler's barrier would wait for
      // every load in flight.)
      asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((S - 2) * (kLoadsA + kLoadsB)) : "memory");
      fetch(q + S - 1, stage<(I + S - 1) % S>());
      if (KG == 1 || q * KG + kg < pieces) compute(stage<I>());
    };
    for_stages([&](auto at) {
      constexpr int I = decltype(at)::value;
      if constexpr (I < S - 1) fetch(I, stage<I>());
    });
    const int32_t steps = (pieces + KG - 1) / KG;
    for (int32_t q = 0; q < steps; q += S)
      for_stages([&](auto at) {
        if (q + decltype(at)::value < steps) step(q + decltype(at)::value, at);
      });
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    if constexpr (KG > 1) {
      static_assert((KG - 1) * FM * FN * 16 * kThreads <= KG * kStage, "the groups' sums in a stage");
      acc_t* m = (acc_t*)stage<0>();
      __syncthreads();
      if (kg > 0) {
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
          for (int j = 0; j < FN; ++j) m[((kg - 1) * FM * FN + i * FN + j) * kThreads + t] = acc[i][j];
      }
      __syncthreads();
      if (kg == 0) {
#pragma unroll
        for (int k = 0; k < KG - 1; ++k)
#pragma unroll
          for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j) acc[i][j] += m[(k * FM * FN + i * FN + j) * kThreads + t];
      }
    }
  }
};

// The tiles in use, kTileKinds of mm_plan.h.
template <int TM_, int TN_, int WM_, int WN_, int S_, int KG_ = 1>
struct TileShape {
  static constexpr int TM = TM_, TN = TN_, WM = WM_, WN = WN_, S = S_, KG = KG_;
  static constexpr int kThreads = 64 * WM * WN * KG;  // of the workgroup
  template <Prod P>
  using Tile = MmaTile<P, TM, TN, WM, WN, S, KG>;
};
template <class F>
dfp_status with_tile(int32_t kind, F f) {
  switch (kind) {
    case 0: return f(TileShape<256, 256, 4, 2, 2>());
    case 1: return f(TileShape<192, 192, 4, 2, 2>());
    case 2: return f(TileShape<192, 128, 4, 2, 2>());
    case 3: return f(TileShape<128, 128, 2, 2, 2>());
    case 4: return f(TileShape<96, 96, 2, 3, 3>());
    case 5: return f(TileShape<64, 64, 2, 2, 3>());
    case 6: return f(TileShape<64, 64, 2, 2, 3, 2>());
    case 7: return f(TileShape<128, 128, 2, 2, 2, 2>());
    default: return f(TileShape<96, 96, 2, 3, 3, 2>());
  }
}

// Consecutive workgroups go round the 8 XCDs, each with an L2 of its own: this turns
// a workgroup's number into one that is consecutive within an XCD, so that the
// tiles an XCD has in flight share operand rows.
__device__ __forceinline__ uint32_t xcd_order(uint32_t id, uint32_t total) {
  const uint32_t xcd = id & 7, q = total >> 3, rem = total & 7;
  return xcd * q + min(xcd, rem) + (id >> 3);
}
// Tile t of tm x tn, walked in bands of `band` tile rows.
__device__ __forceinline__ void tile_of(uint32_t t, uint32_t tm, uint32_t tn, uint32_t band, uint32_t* im,
                                        uint32_t* in) {
  const uint32_t per = band * tn, b = t / per, first = b * band, h = min(band, tm - first), w = t - b * per;
  *im = first + w % h;
  *in = w / h;
}
// Tile (i, j), i <= j, of the upper triangle of n tiles a side, in such bands.
__device__ __forceinline__ void tri_tile_of(uint32_t t, uint32_t n, uint32_t band, uint32_t* im, uint32_t* in) {
  uint32_t first = 0, h, corner;
  for (;;) {
    h = min(band, n - first);
    corner = h * (h + 1) / 2;
    const uint32_t count = corner + h * (n - first - h);
    if (t < count) break;
    t -= count;
    first += h;
  }
  if (t < corner) {
    uint32_t c = 0;
    while (t > c) t -= ++c;  // column c of the corner has c + 1 tiles
    *im = first + t;
    *in = first + c;
  } else {
    t -= corner;
    *im = first + t % h;
    *in = first + h + t / h;
  }
}

}  // namespace dfp
