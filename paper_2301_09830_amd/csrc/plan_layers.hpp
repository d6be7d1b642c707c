// Plan of the linear and gated layers, on the host: which form a call takes, its
// tiles and parts of K, and its workspace.  Sizes, types, alignment and what is
// asked for decide; no device code, and nothing that touches the device.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>

#include "host.hpp"
#include "layer_tiles.hpp"
#include "optcc.h"

namespace occ {

constexpr size_t kWsAlign = 256;        // of the workspace and of each region in it
constexpr size_t kWsHeader = 256;       // the compressor's numeric flags, left alone
constexpr int64_t kMaxTokens = (int64_t)1 << 30;
constexpr int64_t kMaxWidth = (int64_t)1 << 24;   // of in and out
constexpr int64_t kMaxRowBytes = (int64_t)1 << 26;  // of a caller's operand
// The rows of an operand that a wave brings into LDS are addressed from the
// first of them in 31 bits: 32 rows with the 256 x 256 tile, 16 and 8 with the
// others.  So the larger tile takes rows of up to 2^26 bytes (bf16 layers, and
// fp32 ones as planes), the smaller ones of 2^27: dZ of a gated fp32 layer
// (largest_tile).
static_assert(kMaxRowBytes * 32 <= (int64_t)1 << 31 && 2 * kMaxWidth * 2 * 32 <= (int64_t)1 << 31 &&
              2 * kMaxWidth * 4 * 16 <= (int64_t)1 << 31, "offsets of a wave's rows");

inline int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b * b; }
inline int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Regions of a workspace, in order.
struct Carve {
  size_t end = kWsHeader;
  size_t take(size_t bytes) {
    const size_t at = end;
    end += (size_t)up((int64_t)bytes, kWsAlign);
    return at;
  }
  size_t total() const { return end == kWsHeader ? 0 : end; }
};

inline bool ld_ok(int64_t cols, int64_t ld) { return ld >= cols && ld < kMaxDim; }

// ----------------------------------------------------------------------------
// plan of one tiled product
// ----------------------------------------------------------------------------
// Three tiles: 256 x 256 moves the fewest bytes per product, 128 x 128 and
// 64 x 64 leave fewer CUs idle when the result is small.  K is split, and the
// parts joined by a second kernel, where even the small tiles do not fill the
// chip.  The choice is the one of least estimated time: a block's length is
// its K tiles times the measured time of one, plus a fixed part (launch, first
// loads, results); blocks go to the CUs in rounds.
enum Tile { TILE_256, TILE_128, TILE_64, TILE_NUM };

struct TileTimes {
  int side;
  int resident;                    // blocks a CU that do not slow each other down (bf16)
  double k_bf16, k_f32, fixed;     // us; K tiles of all resident blocks
};
// bf16: 8192 x 8192 x K, slope and intercept; 128 and 64: one round at K = 4096.
// fp32 is bound by the matrix unit in each (256 x 256 x 32 in 16384 clocks), so
// two resident blocks share its time.
constexpr TileTimes kTiles[TILE_NUM] = {{256, 1, 1.38, 7.9, 13.0}, {128, 1, 0.57, 2.0, 4.0}, {64, 2, 0.42, 0.58, 3.0}};
constexpr double kJoinUs = 6.0, kJoinBytesPerUs = 5e6;
constexpr int kCUs = 256;
constexpr int kSplits = 8;
constexpr int kSplitCounts[kSplits] = {1, 2, 3, 4, 6, 8, 12, 16};
constexpr double kMaxPartBytes = 512e6;
// A launch holds fewer than 2^32 threads: of blocks of 512, those of the
// products and, beside them, of the bias gradient (16 columns or more each).
constexpr int64_t kMaxBlocks = (((int64_t)1 << 32) - 1) / 512 - kMaxWidth / 16;

// One product of m x width results over k: its blocks with a tile and a split.
struct Product {
  int64_t tiles_m = 0, tiles_n = 0, tiles_k = 0;
  int splits = 1, k_per_split = 1;
  double block_us = 0.0;
  size_t part_bytes = 0;
  int64_t blocks() const { return tiles_m * tiles_n * splits; }
};

// pair: columns come in pairs of rows of W (gated), so a tile makes half as many
// planes: fp32 operands as bf16 planes, K once for each pair of them
inline Product make_product(int64_t m, int64_t width, int64_t k, size_t es, const TileTimes& t, int splits, bool pair, bool planes) {
  Product p;
  p.tiles_m = div_up(m, t.side);
  p.tiles_n = pair ? div_up(width / 2, t.side / 2) : div_up(width, t.side);
  p.tiles_k = div_up(k, kRowBytes / (int64_t)es) * (planes ? kPairs : 1);
  p.k_per_split = (int)div_up(p.tiles_k, splits);
  p.splits = (int)div_up(p.tiles_k, p.k_per_split);
  p.block_us = (double)p.k_per_split * (es == 2 ? t.k_bf16 : t.k_f32) + t.fixed;
  if (p.splits > 1) {
    const double part = (double)p.splits * (double)m * (double)(pair ? 2 * up(width / 2, 4) : up(width, 4)) * 4.0;
    p.part_bytes = (size_t)part;
  }
  return p;
}

inline bool product_fits(const Product& p) {
  return p.blocks() <= kMaxBlocks && p.tiles_k < ((int64_t)1 << 28) && (double)p.part_bytes <= kMaxPartBytes;
}

struct ProductPlan {
  Tile tile = TILE_256;
  Product x, w;   // of the backward pass; the forward pass has x alone
  double us = INFINITY;
  bool fits = false;
};

// Time of a launch on `slots` resident blocks: the blocks of x, then those of
// w, each to the first free slot.  halves: a block of w lands beside one of x
// on the same CU and each runs at half speed.
inline double launch_us(const Product& x, const Product& w, int64_t slots, bool halves) {
  const int64_t nx = x.blocks(), nw = w.blocks();
  const int64_t rest = nx % slots, free = slots - rest;
  const double full = (double)(nx / slots) * x.block_us;   // whole rounds of x
  if (!rest) return full + (double)div_up(nw, slots) * w.block_us;
  if (!nw) return full + x.block_us;
  if (halves && rest + nw > slots)
    return full + x.block_us + 0.5 * (double)nw * w.block_us / ((double)slots - 0.5 * (double)rest);
  const int64_t beside = (int64_t)(x.block_us / w.block_us);   // rounds of w beside the last blocks of x
  const int64_t left = nw - beside * free;
  if (left <= 0) return full + std::max(x.block_us, (double)div_up(nw, free) * w.block_us);
  if (left <= free) return full + std::max(x.block_us, (double)(beside + 1) * w.block_us);
  return full + x.block_us + (double)div_up(left - free, slots) * w.block_us;
}

// Up to two products of one launch, with the same of the given tiles, from the
// first-th on.  m, width, k: of each (m = 0: not there).
inline ProductPlan plan_products(const int64_t (&m)[2], const int64_t (&width)[2], const int64_t (&k)[2], size_t es,
                                 bool pair, bool planes = false, int first = TILE_256,
                                 const TileTimes* tiles = kTiles, int num = TILE_NUM) {
  ProductPlan best;
  for (int t = first; t < num; ++t) {
    const bool halves = es == 4 && tiles[t].resident > 1;
    const int64_t slots = (int64_t)kCUs * (es == 4 ? 1 : tiles[t].resident);
    Product of[2][kSplits];
    int n[2] = {0, 0};
    for (int i = 0; i < 2; ++i) {
      if (!m[i]) {
        of[i][n[i]++] = Product{};
        continue;
      }
      for (const int s : kSplitCounts) {
        const Product p = make_product(m[i], width[i], k[i], es, tiles[t], s, pair, planes);
        if (p.splits != s || (s > 1 && p.k_per_split < 4) || !product_fits(p)) break;
        of[i][n[i]++] = p;
        if (p.blocks() > 2 * slots) break;   // parts of K would only add work
      }
    }
    for (int x = 0; x < n[0]; ++x) {
      for (int w = 0; w < n[1]; ++w) {
        const Product &px = of[0][x], &pw = of[1][w];
        if (px.blocks() + pw.blocks() > kMaxBlocks) continue;
        const double parts = (double)(px.part_bytes + pw.part_bytes);
        const double us = launch_us(px, pw, slots, halves) + (parts > 0.0 ? kJoinUs + parts / kJoinBytesPerUs : 0.0);
        if (us < best.us) {
          best.tile = (Tile)t;
          best.x = px;
          best.w = pw;
          best.us = us;
          best.fits = true;
        }
      }
    }
  }
  return best;
}

// The direct form: 64 x 64 tiles whose operands come through registers, at any
// alignment, dZ made on the way by every block that reads it.  No launch
// before the products, but more work in each of their K tiles: two resident
// blocks 0.50 us in bf16, 1.17 with relu, 1.87 with gelu, 1.02 to 1.31 with
// rows off 16 bytes (the tiles above: 0.42), bound by the VALU, so that a block
// alone takes half of it.  Linear backward, bf16: 94 x 768 x 64 with gelu 8.2 us,
// with dZ made before the products 12.7; 4293 x 463 x 663 with relu 131 us
// against 29.
inline ProductPlan plan_direct(const int64_t (&m)[2], const int64_t (&width)[2], const int64_t (&k)[2], size_t es, bool pair,
                        bool dz, bool act, bool off_pieces) {
  const bool costly = dz && act;   // more than a comparison an element
  const bool back = m[1] || dz;
  const TileTimes t = {64, 1, 0.30 + (costly ? 0.65 : dz ? 0.35 : 0.0) + (off_pieces ? (back ? 0.4 : 0.1) : 0.0),
                       0.56 + (costly ? 0.4 : dz ? 0.2 : 0.0) + (off_pieces ? (back ? 0.15 : 0.06) : 0.0), 3.0};
  return plan_products(m, width, k, es, pair, false, 0, &t, 1);
}

// us to write an operand as planes: 4 bytes of each element are read, 6 written
inline double planes_us(double elements) { return elements * 10.0 / 4e6; }

// An operand the tiled product cannot take in place: rows off 16 bytes, rows
// that end inside a piece, or rows too far apart.
inline bool needs_copy(const void* p, int64_t ld, int64_t cols, size_t es) {
  return !aligned(p, 16) || (size_t)ld * es % 16 || (size_t)cols * es % 16 || ld * (int64_t)es >= kMaxRowBytes;
}

inline int64_t piece_ld(int64_t cols, size_t es) { return up(cols, 16 / (int64_t)es); }

// ----------------------------------------------------------------------------
// forward
// ----------------------------------------------------------------------------
// Up to kFewTokens the weights can be streamed through registers: row by row
// along K up to kDotTokens (one token, 8192 x 8192 bf16: 23.6 us; through the
// matrix instructions 31.6), by matrix instructions above (8 tokens, 4096 x
// 16384: 31.4 us; row by row 36.7).  Above kDotTokens the tiled product takes
// over where it is estimated to be faster: 8192 x 8192 bf16 with 8 tokens 24.6
// against 32.0 us and with 64 tokens 26.1 against 74.8, but 4096 x 4096 with 8
// tokens 13.5 (two launches) against 8.6.
constexpr int64_t kDotTokens = 4;
constexpr int64_t kFewTokens = 64;

// us of the streaming form: a block reads 16 rows of W (of each projection),
// and the more tokens it holds the slower; bf16 rows off 16 bytes take twice as long.
inline double few_us(int64_t tokens, int64_t n_in, int64_t out, size_t es, bool gated, bool on_pieces) {
  const double bytes = (double)div_up(div_up(out, 16), kCUs) * 16.0 * (gated ? 2 : 1) * (double)n_in * (double)es;
  const double rate = 20e3 / (1.0 + (double)tokens / 40.0);   // bytes a us of one CU
  return 2.0 + bytes / rate * (on_pieces || es == 4 ? 1.0 : 2.0);
}

// us of the copy of an operand that the tiled product cannot take in place
inline double copy_us(int64_t rows, int64_t cols, size_t es) { return 3.0 + 2.0 * (double)rows * (double)cols * (double)es / 6e6; }

// us of the launch that makes dZ, sums bias strips or copies operands:
// `elements` read and written
inline double prep_us(double elements, size_t es) { return elements > 0.0 ? 5.0 + elements * (double)es / 5e6 : 0.0; }

// Up to kBiasTokens the bias gradient is summed from dY and Z themselves, in
// blocks beside the products' (a rule on the tokens alone, so that its order
// does not depend on what else a call makes).  bf16, 2048 x 2048, strips and
// direct: 512 tokens 24 and 21 us, 1024 tokens 29 and 26, 2048 tokens 48 and 50;
// with GELU 27 and 27, 33 and 35, 53 and 66.
constexpr int64_t kBiasTokens = 1024;

struct FwdPlan {
  bool few = false, copy_x = false, copy_w = false;
  bool planes = false;   // fp32 on the bf16 matrix units
  bool direct = false;   // operands as they lie, through registers
  size_t x_off = 0, w_off = 0, part_off = 0, bytes = 0;
  ProductPlan prod;
};

inline occ_status_t check_fwd(const occ_linear_t* l, bool gated) {
  if (!l) return OCC_E_NULL;
  if (l->dtype != OCC_F32 && l->dtype != OCC_BF16) return OCC_E_DTYPE;
  if (l->act < OCC_ACT_NONE || l->act > OCC_ACT_SILU) return OCC_E_VALUE;
  if (l->tokens < 0 || l->tokens >= kMaxTokens || l->in < 1 || l->in > kMaxWidth || l->out < 1 || l->out > kMaxWidth)
    return OCC_E_SHAPE;
  const int64_t wide = gated ? 2 * l->out : l->out;
  if (!ld_ok(l->in, l->ldx) || !ld_ok(l->in, l->ldw) || !ld_ok(l->out, l->ldy)) return OCC_E_SHAPE;
  if ((l->R && !ld_ok(l->out, l->ldr)) || (l->Z && !ld_ok(wide, l->ldz))) return OCC_E_SHAPE;
  return OCC_OK;
}

inline occ_status_t plan_fwd(const occ_linear_t& l, bool gated, FwdPlan& f) {
  if (l.tokens == 0) return OCC_OK;
  f.few = l.tokens <= kDotTokens;
  if (f.few) return OCC_OK;
  const size_t es = elem_size(l.dtype);
  const int64_t wide = gated ? 2 * l.out : l.out;
  f.copy_x = needs_copy(l.X, l.ldx, l.in, es);
  f.copy_w = needs_copy(l.W, l.ldw, l.in, es);
  f.prod = plan_products({l.tokens, 0}, {wide, 0}, {l.in, 0}, es, gated);
  const double copies = f.copy_x || f.copy_w ? copy_us(l.tokens * f.copy_x + wide * f.copy_w, l.in, es) : 0.0;
  double tiled = f.prod.us + copies;
  if (copies > 0.0) {
    const ProductPlan p = plan_direct({l.tokens, 0}, {wide, 0}, {l.in, 0}, es, gated, false, false, true);
    if (p.fits && p.us < tiled) {
      f.prod = p;
      tiled = p.us;
      f.direct = true;
      f.copy_x = f.copy_w = false;
    }
  }
  if (l.tokens <= kFewTokens) {
    f.few = few_us(l.tokens, l.in, l.out, es, gated, !needs_copy(l.W, l.ldw, l.in, es)) <= tiled;
    if (f.few) return OCC_OK;
  }
  if (l.dtype == OCC_F32) {
    const ProductPlan p = plan_products({l.tokens, 0}, {wide, 0}, {l.in, 0}, 2, gated, true);
    if (p.fits && p.us + 3.0 + planes_us((double)(l.tokens + wide) * (double)l.in) < tiled) {
      f.prod = p;
      f.direct = false;
      f.planes = f.copy_x = f.copy_w = true;
    }
  }
  if (!f.prod.fits) return OCC_E_SHAPE;
  Carve c;
  const size_t row = f.planes ? (size_t)piece_ld(l.in, 2) * 2 * kPlanes : (size_t)piece_ld(l.in, es) * es;
  if (f.copy_x) f.x_off = c.take((size_t)l.tokens * row);
  if (f.copy_w) f.w_off = c.take((size_t)wide * row);
  if (f.prod.x.splits > 1) f.part_off = c.take(f.prod.x.part_bytes);
  f.bytes = c.total();
  return OCC_OK;
}

// ----------------------------------------------------------------------------
// backward
// ----------------------------------------------------------------------------
struct BwdPlan {
  bool has_dz = false;    // dZ is made (else it is dY)
  bool planes = false;    // fp32 on the bf16 matrix units
  bool direct = false;    // operands as they lie, dZ made where it is loaded
  bool strip_bias = false;   // bias sums by strips of rows, beside dZ
  bool copy_dy = false, copy_x = false, copy_w = false;
  int64_t strip = 0, strips = 0;
  size_t dz_off = 0, bias_off = 0, x_off = 0, w_off = 0, dx_part = 0, dw_part = 0, bytes = 0;
  int64_t ldd = 0;
  ProductPlan prod;
};

inline occ_status_t check_bwd(const occ_linear_grad_t* l, bool gated) {
  if (!l) return OCC_E_NULL;
  if (l->dtype != OCC_F32 && l->dtype != OCC_BF16) return OCC_E_DTYPE;
  if (l->dw_dtype != l->dtype && l->dw_dtype != OCC_F32) return OCC_E_DTYPE;
  if (l->act < OCC_ACT_NONE || l->act > OCC_ACT_SILU) return OCC_E_VALUE;
  if (l->tokens < 0 || l->tokens >= kMaxTokens || l->in < 1 || l->in > kMaxWidth || l->out < 1 || l->out > kMaxWidth)
    return OCC_E_SHAPE;
  const int64_t wide = gated ? 2 * l->out : l->out;
  const bool z = gated || l->act != OCC_ACT_NONE;
  if (!l->dX && !l->dW && !l->dbias) return OCC_E_NULL;
  if (!ld_ok(l->out, l->lddy) || (z && !ld_ok(wide, l->ldz))) return OCC_E_SHAPE;
  if (l->dX && (!ld_ok(l->in, l->lddx) || !ld_ok(l->in, l->ldw))) return OCC_E_SHAPE;
  if (l->dW && (!ld_ok(l->in, l->lddw) || !ld_ok(l->in, l->ldx))) return OCC_E_SHAPE;
  return OCC_OK;
}

// Largest tile for a layer whose dZ is `wide` columns of es bytes.  (In fp32 the
// 256 x 256 tile is taken where K is short and results are many, bound by their
// stores: dW alone of 30 x 4096 x 16384 85 us, with 128 x 128 tiles 93.)
inline int largest_tile(int64_t wide, size_t es) {
  return piece_ld(wide, es) * (int64_t)es > kMaxRowBytes ? TILE_128 : TILE_256;
}

inline occ_status_t plan_bwd(const occ_linear_grad_t& l, bool gated, BwdPlan& f) {
  if (l.tokens == 0) return OCC_OK;
  const size_t es = elem_size(l.dtype);
  const int64_t wide = gated ? 2 * l.out : l.out;
  const bool prod = l.dX || l.dW;
  const bool act = gated || l.act != OCC_ACT_NONE;
  f.has_dz = act && prod;
  f.strip_bias = l.dbias && l.tokens > kBiasTokens;
  if (prod) {
    f.copy_dy = !act && needs_copy(l.dY, l.lddy, l.out, es);
    f.copy_w = l.dX && needs_copy(l.W, l.ldw, l.in, es);
    f.copy_x = l.dW && needs_copy(l.X, l.ldx, l.in, es);
    const int64_t m[2] = {l.dX ? l.tokens : 0, l.dW ? wide : 0}, width[2] = {l.in, l.in}, k[2] = {wide, l.tokens};
    f.prod = plan_products(m, width, k, es, false, false, largest_tile(wide, es));
    const double x = l.dW ? (double)l.tokens * (double)l.in : 0.0, w = l.dX ? (double)wide * (double)l.in : 0.0;
    const double dz = (double)l.tokens * (double)wide, dy = (double)l.tokens * (double)l.out;
    const double copied = (f.copy_x ? x : 0.0) + (f.copy_w ? w : 0.0) + (f.copy_dy ? dz : 0.0);
    double us = f.prod.us + prep_us((act ? dy + 2.0 * dz : f.strip_bias ? dy : 0.0) + 2.0 * copied, es);
    if (us > f.prod.us && !f.strip_bias) {
      const bool off_pieces = copied > 0.0 || (act && (needs_copy(l.dY, l.lddy, l.out, es) || needs_copy(l.Z, l.ldz, wide, es)));
      const ProductPlan p = plan_direct(m, width, k, es, false, act, gated || l.act != OCC_ACT_RELU, off_pieces);
      // each product reads dY and Z for itself
      const double all = p.us + (act ? (dy + dz) * (double)es * ((l.dX ? 1 : 0) + (l.dW ? 1 : 0)) / 6e6 : 0.0);
      if (p.fits && all < us) {
        f.prod = p;
        us = all;
        f.direct = true;
        f.has_dz = f.copy_dy = f.copy_x = f.copy_w = false;
      }
    }
    if (l.dtype == OCC_F32) {
      const ProductPlan p = plan_products(m, width, k, 2, false, true);
      // dZ, if it is made, is written as planes in place of fp32
      const double planes = 3.0 + planes_us(x + w + dz) + (act || f.strip_bias ? dy * 4.0 / 5e6 : 0.0);
      if (p.fits && p.us + planes < us) {
        f.prod = p;
        f.planes = true;
        f.direct = false;
        f.has_dz = act;
        f.copy_x = l.dW;
        f.copy_w = l.dX;
        f.copy_dy = !act;
      }
    }
    if (!f.prod.fits) return OCC_E_SHAPE;
  }
  const size_t os = f.planes ? 2 : es, np = f.planes ? kPlanes : 1;   // of operands in the workspace
  f.ldd = piece_ld(wide, os);
  Carve c;
  if (f.has_dz || f.copy_dy) f.dz_off = c.take((size_t)l.tokens * f.ldd * os * np);
  if (f.has_dz || f.strip_bias) {
    // enough blocks to fill the chip several times, whole groups of rows in
    // each; fewer, longer strips where their sums have to be added
    const int64_t across = div_up(l.out, DZ_LANES * 4), most = f.strip_bias ? 2048 : 8192;
    const int64_t down = std::max<int64_t>(1, std::min<int64_t>(div_up(most, across), div_up(l.tokens, DZ_ROWS)));
    f.strip = up(div_up(l.tokens, down), DZ_ROWS);
    f.strips = div_up(l.tokens, f.strip);
    if (across * f.strips >= ((int64_t)1 << 30)) return OCC_E_SHAPE;
    if (f.strip_bias) f.bias_off = c.take((size_t)f.strips * wide * 4);
  }
  if (f.copy_w) f.w_off = c.take((size_t)wide * piece_ld(l.in, os) * os * np);
  if (f.copy_x) f.x_off = c.take((size_t)l.tokens * piece_ld(l.in, os) * os * np);
  if (f.prod.x.splits > 1) f.dx_part = c.take(f.prod.x.part_bytes);
  if (f.prod.w.splits > 1) f.dw_part = c.take(f.prod.w.part_bytes);
  f.bytes = c.total();
  return OCC_OK;
}

}  // namespace occ
