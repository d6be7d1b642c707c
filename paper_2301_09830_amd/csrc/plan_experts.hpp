// Plan of the experts' layers, on the host: form, tiles and workspace, from
// sizes, types, alignment and what is asked for.  The lengths of the experts'
// runs are on the device: estimates take the mean length, launches hold the
// blocks that any lengths may need.
#pragma once

#include "plan_layers.hpp"

namespace occ {

constexpr int64_t kMaxExperts = OCC_MAX_EXPERTS;

// Runs of rows of each expert that at most `rows` rows of `experts` can make,
// `run` rows or fewer each.
inline int64_t most_runs(int64_t rows, int64_t experts, int64_t run) { return rows / run + std::min(rows, experts); }

// The same as expected: experts differ, so that some have a run more than the
// mean's.
inline double mean_runs(int64_t rows, int64_t experts, int64_t run) {
  const double n = (double)std::min(rows, experts), mean = (double)rows / n;
  return n * std::max(1.0, mean / (double)run + (experts > 1 ? 0.6 : 0.5));
}

// Lanes that share a token in the router's gradient, and the tokens of one of
// its launches: a launch holds fewer than 2^32 threads, in whole blocks of 256.
inline int route_lanes(int64_t experts, int k) { return k > 16 || experts > 256 ? 64 : 16; }

inline int64_t route_bwd_part(int64_t experts, int k) {
  return (((int64_t)1 << 32) - 1) / 256 * (256 / route_lanes(experts, k));
}

// A matrix of every expert: rows x cols, ld apart, and `stride` to the next.
inline bool experts_ok(int64_t experts, int64_t rows, int64_t cols, int64_t ld, int64_t stride) {
  if (!ld_ok(cols, ld)) return false;
  return experts == 1 || (stride >= (rows - 1) * ld + cols && stride < ((int64_t)1 << 44) / experts);
}

// us of `blocks` blocks on `slots` places: whole rounds while there are few and
// their number is known, which it is not where lengths are near a run's.
inline double rounds_us(double blocks, int64_t slots, double block_us, bool known) {
  const double r = blocks / (double)slots;
  return (r <= 0.7 ? 1.0 : known ? r < 4.0 ? std::ceil(r) : r : r + 0.5) * block_us;
}

struct ExpertsTile {
  Tile tile = TILE_256;
  double us = INFINITY;
};

// us of one K tile and the fixed part, of a form (the layers' times)
inline double tile_us(const TileTimes& t, size_t es, double k_tiles) {
  return k_tiles * (es == 2 ? t.k_bf16 : t.k_f32) + t.fixed;
}

inline int64_t tile_slots(const TileTimes& t, size_t es) { return (int64_t)kCUs * (es == 4 ? 1 : t.resident); }

// Forms that stream the weights, for few rows of an expert: rows of a run, and
// ns of the whole chip that a block takes, fixed and for each 2 KiB of K
// (linear, gated).  Measured at 64 rows of each of 8 and 64 experts, in 512 to
// 4096; bf16 rows off 16 bytes take 1.5 times as long along K, twice through
// the matrix instructions.  With two rows an expert or fewer they are ahead of
// the tiles (8 experts, 4096 x 4096, gated, 16 rows 78 against 89 us; 3 experts, 1408 x
// 3008, 6 rows 7.4 and 9.3), from some eight on behind (8 experts, 1408 x 3008, 64
// rows 20.1 and 13.5, 512 rows 57 and 18.5; fp32 64 rows 41 and 55, 512 rows 118 and 85).
struct FewTimes {
  int form, run;
  double fixed[2], k[2];
};
constexpr FewTimes kFewForms[4] = {{1, 4, {2.35, 2.35}, {1.35, 1.35}},
                                   {16, 16, {5.1, 8.0}, {6.45, 9.6}},
                                   {32, 32, {3.0, 5.0}, {8.5, 13.0}},
                                   {64, 64, {0.0, 9.5}, {0.0, 18.6}}};

inline int64_t few_across(int form, int64_t out, bool gated) {
  return form == 1 ? div_up(gated ? out : div_up(out, 2), 4) : div_up(out, 16);
}

inline double few_experts_us(const occ_experts_t& p, bool gated, const FewTimes& t, size_t es) {
  const double blocks = mean_runs(p.l.tokens, p.experts, t.run) * (double)few_across(t.form, p.l.out, gated);
  const bool off = es == 2 && needs_copy(p.l.W, p.l.ldw, p.l.in, es);
  const double k = (double)p.l.in * (double)es / 2048.0;
  return 3.0 + blocks * (t.fixed[gated] + t.k[gated] * k) * 1e-3 * (off ? t.form == 1 ? 1.5 : 2.0 : 1.0);
}

struct ExpertsFwdPlan {
  int few = 0;           // 1: along K; 16, 32, 64: rows through the matrix instructions
  bool copy_x = false, copy_w = false, planes = false, direct = false;
  Tile tile = TILE_64;
  int64_t blocks = 0;
  size_t x_off = 0, w_off = 0, bytes = 0;
};

inline occ_status_t check_experts_fwd(const occ_experts_t* p, bool gated) {
  if (!p) return OCC_E_NULL;
  OCC_TRY(check_fwd(&p->l, gated));
  const int64_t wide = gated ? 2 * p->l.out : p->l.out;
  if (p->experts < 1 || p->experts > kMaxExperts) return OCC_E_SHAPE;
  return experts_ok(p->experts, wide, p->l.in, p->l.ldw, p->stride_w) ? OCC_OK : OCC_E_SHAPE;
}

// Rows of 16 bytes that follow each other from one expert to the next.
inline bool experts_copy(const void* p, int64_t ld, int64_t cols, int64_t stride, int64_t experts, size_t es) {
  return needs_copy(p, ld, cols, es) || (experts > 1 && (size_t)stride * es % 16);
}

inline double fwd_tile_us(const occ_experts_t& p, bool gated, const TileTimes& t, size_t es, bool planes) {
  const int64_t tiles_n = gated ? div_up(p.l.out, t.side / 2) : div_up(p.l.out, t.side);
  const double k = (double)div_up(p.l.in, kRowBytes / (int64_t)es) * (planes ? kPairs : 1);
  const double blocks = mean_runs(p.l.tokens, p.experts, t.side) * (double)tiles_n;
  const double mean = (double)p.l.tokens / (double)std::min(p.l.tokens, p.experts) / t.side;
  const bool known = p.experts == 1 || mean < 0.33 || mean > 2.0;
  double block = tile_us(t, es, k);
  // one resident block alone does not share its CU (0.27 us a K tile of 64 x 64)
  if (es == 2 && t.resident > 1 && blocks <= (double)kCUs) block = k * 0.65 * t.k_bf16 + t.fixed;
  return rounds_us(blocks, tile_slots(t, es), block, known);
}

inline ExpertsTile best_fwd(const occ_experts_t& p, bool gated, size_t es, bool planes) {
  ExpertsTile best;
  for (int t = TILE_256; t < TILE_NUM; ++t) {
    const double us = fwd_tile_us(p, gated, kTiles[t], es, planes);
    if (us < best.us) best = {(Tile)t, us};
  }
  return best;
}

inline occ_status_t plan_experts_fwd(const occ_experts_t& p, bool gated, ExpertsFwdPlan& f) {
  const occ_linear_t& l = p.l;
  if (l.tokens == 0) return OCC_OK;
  const size_t es = elem_size(l.dtype);
  const int64_t wide = gated ? 2 * l.out : l.out, used = std::min(l.tokens, p.experts);
  const double mean = (double)l.tokens / (double)used;
  f.copy_x = needs_copy(l.X, l.ldx, l.in, es);
  f.copy_w = experts_copy(l.W, l.ldw, l.in, p.stride_w, p.experts, es);
  ExpertsTile best = best_fwd(p, gated, es, false);
  double us = best.us;
  if (f.copy_x || f.copy_w) {
    us += copy_us(l.tokens * f.copy_x + p.experts * wide * f.copy_w, l.in, es);
    const TileTimes t = {64, 1, 0.40, 0.62, 3.0};
    const double direct = fwd_tile_us(p, gated, t, es, false);
    if (direct < us) {
      f.direct = true;
      f.copy_x = f.copy_w = false;
      best.tile = TILE_64;
      us = direct;
    }
  }
  if (l.dtype == OCC_F32) {
    const ExpertsTile b = best_fwd(p, gated, 2, true);
    const double all = b.us + 3.0 + planes_us((double)(l.tokens + p.experts * wide) * (double)l.in);
    if (all < us) {
      best = b;
      f.direct = false;
      f.planes = f.copy_x = f.copy_w = true;
    }
  }
  // the weights of the experts that have rows are read in any form
  const double weights = (double)used * (double)wide * (double)l.in * (double)es / 5.5e6;
  us = std::max(us + 2.0, weights);
  if (mean <= (double)kFewTokens)
    for (const FewTimes& t : kFewForms) {
      if (t.form == 64 && !gated) continue;   // never ahead of two runs of 32
      const double few = std::max(few_experts_us(p, gated, t, es), weights);
      if (few > us || (f.few && few == us)) continue;
      us = few;
      f.few = t.form;
    }
  if (f.few) {
    f.copy_x = f.copy_w = f.planes = f.direct = false;
    const int run = f.few == 1 ? 4 : f.few;
    f.blocks = most_runs(l.tokens, p.experts, run) * few_across(f.few, l.out, gated);
    return f.blocks <= kMaxBlocks ? OCC_OK : OCC_E_SHAPE;
  }
  f.tile = best.tile;
  const int side = f.direct ? 64 : kTiles[f.tile].side;
  f.blocks = most_runs(l.tokens, p.experts, side) * (gated ? div_up(l.out, side / 2) : div_up(l.out, side));
  if (f.blocks > kMaxBlocks || p.experts * wide >= ((int64_t)1 << 31)) return OCC_E_SHAPE;
  Carve c;
  const size_t row = f.planes ? (size_t)piece_ld(l.in, 2) * 2 * kPlanes : (size_t)piece_ld(l.in, es) * es;
  if (f.copy_x) f.x_off = c.take((size_t)l.tokens * row);
  if (f.copy_w) f.w_off = c.take((size_t)(p.experts * wide) * row);
  f.bytes = c.total();
  return OCC_OK;
}

// Before the products: blocks of 256 threads in a launch of fewer than 2^32,
// beside those of the copies.
constexpr int64_t kMaxPrepBlocks = (((int64_t)1 << 32) - 1) / 256 - 3 * kMaxCopyBlocks;

struct ExpertsBwdPlan {
  bool has_dz = false, planes = false, direct = false;
  bool copy_dy = false, copy_x = false, copy_w = false;
  Tile tile = TILE_64;
  int64_t dx_blocks = 0, dw_blocks = 0;
  int64_t strip = 0, strips = 0, across = 0;   // of dZ and the bias sums
  size_t dz_off = 0, bias_off = 0, x_off = 0, w_off = 0, bytes = 0;
  int64_t ldd = 0;
};

inline occ_status_t check_experts_bwd(const occ_experts_grad_t* p, bool gated) {
  if (!p) return OCC_E_NULL;
  OCC_TRY(check_bwd(&p->l, gated));
  const occ_linear_grad_t& l = p->l;
  const int64_t wide = gated ? 2 * l.out : l.out;
  if (p->experts < 1 || p->experts > kMaxExperts) return OCC_E_SHAPE;
  if (l.dX && !experts_ok(p->experts, wide, l.in, l.ldw, p->stride_w)) return OCC_E_SHAPE;
  if (l.dW && !experts_ok(p->experts, wide, l.in, l.lddw, p->stride_dw)) return OCC_E_SHAPE;
  return OCC_OK;
}

// Tiles of dW of one expert, dealt to 8 XCDs in whole runs.
inline int64_t dw_blocks_of(int64_t wide, int64_t in, int64_t experts, int side) {
  const int64_t tiles = div_up(wide, side) * div_up(in, side);
  return experts * (tiles >= 8 ? up(tiles, 8) : tiles);
}

inline double bwd_tile_us(const occ_experts_grad_t& p, int64_t wide, const TileTimes& t, size_t es, bool planes) {
  const occ_linear_grad_t& l = p.l;
  const int64_t bk = kRowBytes / (int64_t)es, tiles_n = div_up(l.in, t.side);
  const double pairs = planes ? kPairs : 1;
  const double x = l.dX ? mean_runs(l.tokens, p.experts, t.side) * (double)tiles_n : 0.0;
  const double xus = tile_us(t, es, (double)div_up(wide, bk) * pairs);
  const double w = l.dW ? (double)p.experts * (double)div_up(wide, t.side) * (double)tiles_n : 0.0;
  const double wus = tile_us(t, es, ((double)l.tokens / (double)(p.experts * bk) + 0.5) * pairs);
  // the longest expert has twice the mean's rows, and its tiles of dW may end last
  const double longest = p.experts > 1 ? 2.0 * wus - t.fixed : wus;
  const double slots = (double)tile_slots(t, es), sum = (x * xus + w * wus) / slots;
  return std::max({sum, x > 0.0 ? xus : 0.0, w > 0.0 ? longest : 0.0});
}

inline ExpertsTile best_bwd(const occ_experts_grad_t& p, int64_t wide, size_t es, bool planes, int first) {
  ExpertsTile best;
  for (int t = first; t < TILE_NUM; ++t) {
    const double us = bwd_tile_us(p, wide, kTiles[t], es, planes);
    if (us < best.us) best = {(Tile)t, us};
  }
  return best;
}

inline occ_status_t plan_experts_bwd(const occ_experts_grad_t& p, bool gated, ExpertsBwdPlan& f) {
  const occ_linear_grad_t& l = p.l;
  if (l.tokens == 0) return OCC_OK;
  const size_t es = elem_size(l.dtype);
  const int64_t wide = gated ? 2 * l.out : l.out;
  const bool prod = l.dX || l.dW, act = gated || l.act != OCC_ACT_NONE;
  f.has_dz = act && prod;
  if (prod) {
    f.copy_dy = !act && needs_copy(l.dY, l.lddy, l.out, es);
    f.copy_w = l.dX && experts_copy(l.W, l.ldw, l.in, p.stride_w, p.experts, es);
    f.copy_x = l.dW && needs_copy(l.X, l.ldx, l.in, es);
    ExpertsTile best = best_bwd(p, wide, es, false, largest_tile(wide, es));
    const double x = l.dW ? (double)l.tokens * (double)l.in : 0.0;
    const double w = l.dX ? (double)(p.experts * wide) * (double)l.in : 0.0;
    const double dz = (double)l.tokens * (double)wide, dy = (double)l.tokens * (double)l.out;
    const double copied = (f.copy_x ? x : 0.0) + (f.copy_w ? w : 0.0) + (f.copy_dy ? dz : 0.0);
    const double bias = l.dbias ? dy + (act ? dz : 0.0) : 0.0;
    double us = best.us + prep_us((act ? dy + 2.0 * dz : bias) + 2.0 * copied, es);
    if (f.has_dz || copied > 0.0) {
      const bool off = copied > 0.0 || (act && (needs_copy(l.dY, l.lddy, l.out, es) || needs_copy(l.Z, l.ldz, wide, es)));
      const bool costly = gated || l.act > OCC_ACT_RELU;
      const TileTimes t = {64, 1, 0.30 + (act ? (costly ? 0.65 : 0.35) : 0.0) + (off ? 0.4 : 0.0),
                           0.56 + (act ? (costly ? 0.4 : 0.2) : 0.0) + (off ? 0.15 : 0.0), 3.0};
      const double again = act ? (dy + dz) * (double)es * ((l.dX ? 1 : 0) + (l.dW ? 1 : 0)) / 6e6 : 0.0;
      const double direct = bwd_tile_us(p, wide, t, es, false) + again + prep_us(bias, es);
      if (direct < us) {
        f.direct = true;
        f.has_dz = f.copy_dy = f.copy_x = f.copy_w = false;
        best.tile = TILE_64;
        us = direct;
      }
    }
    if (l.dtype == OCC_F32) {
      const ExpertsTile b = best_bwd(p, wide, 2, true, TILE_256);
      const double planes = 3.0 + planes_us(x + w + dz) + (act || l.dbias ? dy * 4.0 / 5e6 : 0.0);
      if (b.us + planes < us) {
        best = b;
        f.planes = true;
        f.direct = false;
        f.has_dz = act;
        f.copy_x = l.dW;
        f.copy_w = l.dX;
        f.copy_dy = !act;
      }
    }
    f.tile = best.tile;
    const int side = f.direct ? 64 : kTiles[f.tile].side;
    if (l.dX) f.dx_blocks = up(most_runs(l.tokens, p.experts, side) * div_up(l.in, side), 8);
    if (l.dW) f.dw_blocks = dw_blocks_of(wide, l.in, p.experts, side);
    if (f.dx_blocks + f.dw_blocks > kMaxBlocks || p.experts * wide >= ((int64_t)1 << 31)) return OCC_E_SHAPE;
  }
  const int64_t bias_blocks = l.dbias ? p.experts * div_up(wide, 64) : 0;   // of the products' launch
  if (bias_blocks > kMaxBlocks / 2 || f.dx_blocks + f.dw_blocks + bias_blocks > (((int64_t)1 << 32) - 1) / 512)
    return OCC_E_SHAPE;
  const size_t os = f.planes ? 2 : es, np = f.planes ? kPlanes : 1;   // of operands in the workspace
  f.ldd = piece_ld(wide, os);
  Carve c;
  if (f.has_dz || f.copy_dy) f.dz_off = c.take((size_t)l.tokens * f.ldd * os * np);
  if (f.has_dz || l.dbias) {
    // enough blocks to fill the chip several times; longer strips where their sums have to be added
    f.across = div_up(l.out, DZ_LANES * 4);
    const int64_t most = l.dbias ? 2048 : 8192;
    const int64_t down = std::max<int64_t>(1, std::min<int64_t>(div_up(most, f.across), div_up(l.tokens, DZ_ROWS)));
    f.strip = up(div_up(l.tokens, down), DZ_ROWS);
    f.strips = most_runs(l.tokens, p.experts, f.strip);
    if (f.across * f.strips > kMaxPrepBlocks) return OCC_E_SHAPE;
    if (l.dbias) f.bias_off = c.take((size_t)f.strips * wide * 4);
  }
  if (f.copy_w) f.w_off = c.take((size_t)(p.experts * wide) * piece_ld(l.in, os) * os * np);
  if (f.copy_x) f.x_off = c.take((size_t)l.tokens * piece_ld(l.in, os) * os * np);
  f.bytes = c.total();
  return OCC_OK;
}

}  // namespace occ
