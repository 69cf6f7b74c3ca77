// Which kernel, tiles and slices the products of the INT8 linear layers and of the orthogonalised updates take:
// host arithmetic of every call, without any of HIP.
#pragma once

#include <algorithm>
#include <cstdint>

namespace dfp {

constexpr int kPiece = 128;  // bytes of an operand row per step of the tile loop (mma_tile.h)
inline int64_t i8_ld(int64_t cols) { return (cols + 127) / 128 * 128; }

// The tiles in use and an estimate of a product's time (us), from products of 64 to 1024
// tiles (`tiles` / 256 rounded up: the most a CU has) at reductions of 32 and 96 pieces:
//   start + (rounds - 1) start_round + pieces (piece, from 128 to 256 tiles rising to
//   piece_full, + (rounds - 1) piece_round)
// for I8 and F16, and for F16X2.  Outputs of a tile per time rise with its side, but so
// does what starts and ends it, and 256 CUs are filled in steps.
struct TileCost {
  double start, start_round, piece, piece_full, piece_round;
};
struct TileKind {
  int32_t tm, tn;
  TileCost cost[2];
};
constexpr TileKind kTileKinds[] = {
    {256, 256, {{14.0, 12.5, 1.23, 1.61, 1.60}, {14.5, 13.0, 1.55, 2.14, 2.12}}},
    {192, 192, {{8.6, 7.0, 0.77, 0.96, 0.95}, {8.5, 7.5, 0.96, 1.29, 1.25}}},
    {192, 128, {{5.5, 5.5, 0.71, 0.76, 0.58}, {6.8, 5.0, 0.70, 0.92, 0.80}}},
    {128, 128, {{5.0, 4.0, 0.63, 0.63, 0.41}, {6.0, 4.0, 0.61, 0.67, 0.56}}},
    {96, 96, {{4.0, 2.3, 0.35, 0.37, 0.36}, {4.5, 2.3, 0.39, 0.43, 0.44}}},
    {64, 64, {{1.0, 1.8, 0.28, 0.30, 0.16}, {1.7, 1.4, 0.29, 0.30, 0.17}}},
    {64, 64, {{2.3, 2.2, 0.20, 0.21, 0.20}, {3.1, 2.5, 0.20, 0.22, 0.21}}},     // two groups each
    {128, 128, {{6.5, 5.0, 0.47, 0.53, 0.51}, {7.5, 6.5, 0.49, 0.59, 0.60}}},
    {96, 96, {{5.5, 4.0, 0.30, 0.29, 0.31}, {6.5, 4.3, 0.30, 0.33, 0.36}}},
};
constexpr int kTileKindCount = 9;
// slow: what the reduction takes more when operands come from memory.
inline double tile_us(const TileKind& k, bool split, int64_t tiles, int64_t pieces, double slow = 1.) {
  const TileCost& c = k.cost[split];
  const double more = (double)((tiles + 255) / 256 - 1);
  const double full = tiles >= 256 ? 1. : tiles <= 128 ? 0. : (double)(tiles - 128) / 128.;
  return c.start + more * c.start_round +
         (double)pieces * slow * (c.piece + full * (c.piece_full - c.piece) + more * c.piece_round);
}

// ------------------------------------------------------------ INT8 products
// The kernel of a product by an estimate of its time (us).
//   k_few    a CU takes 0.15, 0.21 or 0.35 for a piece of 16 columns by up to 16, 32
//            or 64 rows (4096 x 4096, 8192 x 2048 and 8192 x 8192 weights).
//   k_tiles  tile_us; with weights that come from memory, as they do for few rows, a
//            quarter more.  Slices mean that their sums are written and read (4 TB/s)
//            and a second kernel (4).
// At 64 rows: 4096 x 4096 k_few 13.8, tiles 12.0; 8192 x 2048 13.4 and 8.2; 8192 x
// 8192 44.7 and 22.1; 1024 x 1024 5.0 and 5.1.  At 24: 9.7 and 10.0; 8.6 and 7.3; 25.4 and
// 20.4; 3.5 and 4.7.  At 16, where k_few runs always: 7.9 and 9.7; 7.0 and 7.0; 19.4 and
// 20.3; 3.2 and 4.5.
constexpr int32_t kFewRows = 64;
constexpr int64_t kMostI8PartBytes = 64 << 20;

struct I8Plan {
  int32_t kind;         // of tile; -1: the kernel for few rows
  int32_t slices, per;  // of the reduction, pieces in each
  int64_t bytes;        // the slices' sums
};
inline I8Plan plan_gemm_i8(int64_t m, int64_t n, int64_t k) {
  I8Plan best{-1, 1, 0, 0};
  const int64_t pieces = i8_ld(k) / kPiece;
  double least = 1e30;
  if (m <= kFewRows) {
    least = 2. + ((n + 15) / 16 + 255) / 256 * pieces * (m <= 16 ? 0.15 : m <= 32 ? 0.21 : 0.35);
    if (m <= 16) return best;
  }
  for (int t = 0; t < kTileKindCount; ++t) {
    const TileKind& kind = kTileKinds[t];
    const int64_t tiles = ((m + kind.tm - 1) / kind.tm) * ((n + kind.tn - 1) / kind.tn);
    for (int64_t slices = 1; slices <= 16 && slices <= pieces; slices *= 2) {
      const int64_t per = (pieces + slices - 1) / slices, used = (pieces + per - 1) / per;
      const int64_t bytes = used > 1 ? used * m * n * 4 : 0;
      if (bytes > kMostI8PartBytes) break;
      double us = tile_us(kind, false, tiles * used, per, m <= kFewRows ? 1.25 : 1.);
      if (used > 1) us += 4. + 2. * bytes / 4e6;
      if (us < least) {
        least = us;
        best = {t, (int32_t)used, (int32_t)per, bytes};
      }
    }
  }
  return best;
}

// ---------------------------------------------------- orthogonalised updates
// A product's tiles and slices by an estimate of its time: tile_us and 2 us a round for
// 128 x 128 outputs (which are stored twice, after another pass through LDS); slices
// mean that their sums are written and read (5 TB/s) and a second kernel (4 us).
struct MmPlan {
  int32_t kind, slices, per;
  int64_t bytes;
  double us;
};
constexpr int64_t kMostMmPartBytes = 128 << 20;

// Tiles of the symmetric products: square, and of two parts not 96 x 96 by one group,
// which two groups always beat (kTileKinds[4] and [8]).
constexpr bool has_triangle(int kind, bool split) {
  return kTileKinds[kind].tm == kTileKinds[kind].tn && !(split && kind == 4);
}

inline MmPlan plan_mm(int64_t m, int64_t n, int64_t pieces, int64_t batch, bool symmetric, bool sliceable, bool split) {
  MmPlan best{};
  double least = 1e30;
  for (int t = 0; t < kTileKindCount; ++t) {
    const TileKind& kind = kTileKinds[t];
    if (symmetric && !has_triangle(t, split)) continue;
    const int64_t tm = (m + kind.tm - 1) / kind.tm, tn = (n + kind.tn - 1) / kind.tn;
    const int64_t tiles = (symmetric ? tm * (tm + 1) / 2 : tm * tn) * batch;
    for (int64_t s = 1; s <= (sliceable ? 32 : 1) && s <= pieces; ++s) {
      const int64_t per = (pieces + s - 1) / s, used = (pieces + per - 1) / per;
      if (used != s) continue;
      const int64_t bytes = s > 1 ? s * tiles * kind.tm * kind.tn * 4 : 0;
      if (bytes > kMostMmPartBytes) break;
      double us = tile_us(kind, split, tiles * s, per) +
                  2. * ((tiles * s + 255) / 256) * kind.tm * kind.tn / 16384.;
      if (s > 1) us += 4. + 2. * bytes / 5e6;
      if (us < least) {
        least = us;
        best = {t, (int32_t)s, (int32_t)per, bytes, us};
      }
    }
  }
  return best;
}

// The three products of an iteration on [rows][cols], padded to 64, of a batch; split: operands of two f16 numbers.
struct OrthoPlan {
  MmPlan gram, poly, step;
  bool grouped;  // weight steps: iterations on the small side (3 us a launch)
};
inline OrthoPlan plan_ortho(int64_t batch, int64_t rows, int64_t cols, bool split) {
  const int64_t Rp = (rows + 63) / 64 * 64, Cp = (cols + 63) / 64 * 64, rp = std::min(Rp, Cp), longer = std::max(Rp, Cp);
  const int64_t per_piece = split ? 32 : 64;
  OrthoPlan p;
  // (only the Gram product has reductions longer than its sides)
  p.gram = plan_mm(rp, rp, longer / per_piece, batch, true, true, split);
  p.poly = plan_mm(rp, rp, rp / per_piece, batch, true, false, split);
  p.step = plan_mm(Rp, Cp, rp / per_piece, batch, false, false, split);
  p.grouped = split && p.gram.us + p.step.us > 3. * p.poly.us + 3.;
  return p;
}

}  // namespace dfp
