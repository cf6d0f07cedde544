// Internal declarations of the gated feed-forward block: its products in fp32,
// bf16 and 8-bit codes, checkpoints in 8 bits, and the row kernels around them.
#pragma once

#include "vocab_internal.h"

namespace hfk {

enum { GA_SIGMOID, GA_TANH, GA_RELU, GA_SILU, GA_GELU, GA_GELU_TANH };
enum { KEEP_NONE, KEEP_FULL, KEEP_CODES };

// Columns of a checkpoint that share a scale byte.
constexpr int CODE_BLOCK = 32;
// Widths of packed codes: whole K blocks of 128.
constexpr int CPAD = 128;

// C(m, n) = sum_k A(m, k) B(n, k), m contiguous in the output (see mfma_tile.h).
struct GGemm {
  int M, N, K;
  int m0;                // columns of the output before it are another launch's
  const void *A, *A1, *B;
  long long lda, lda1, ldb;   // lda1: of A1 for few rows (else A's)
  int alim, blim;        // rows m of A and n of B that exist, where these are rows
  int kh;                // row products: A1 has the rows k from kh on
  // operands whose rows are k: those from ktail on are read here, where zeros
  // follow the last one; null: they follow where the operand is
  const void *at, *bt;
  long long ldat, ldbt;
  int ktail;
  int splits, tile;
};

// output tiles of a product's columns from m0 on
inline int gated_tiles(const GGemm& g) {
  const int rm = tile_m(g.tile), rn = tile_n(g.tile);
  return g.M > g.m0 && g.N > 0 ? (g.M - g.m0 + rm - 1) / rm * ((g.N + rn - 1) / rn) : 0;
}

struct GEpi {
  int act, F, Fp;        // hidden width, and as the workspace has it
  int T;                 // rows of the call
  void* h;               // phi(g) u: fp32 for codes, else of the type
  long long ldh;
  int h32;               // few rows: h is fp32 whatever the type
  int dup;               // > 0: the rounding's rest too, dup rows further down
  int keep;
  void* kept;            // g, and F elements further u
  long long ldk;
  uint8_t* ks;           // scale bytes of g's blocks, and then of u's
  long long ldks;
  void* dgu;             // dg, and Fp columns further du
  long long lddgu;
  const float *sn, *sm, *sm1;   // codes: scales of the rows n, and of m (sm1: of u)
  float* hmax;           // codes: largest |h| of a row in each wave's columns
  int ldmax;
  void *out, *out1;      // out1: rows from n1 on, at row n - n1
  long long ldo, ldo1;
  int n1, nout, mout;    // rows of each, columns
  int accumulate;
  float* part;           // partials [split][n][m - m0] (codes: int32), rows ldp apart
  long long ldp;
};

// The kernels with an activation, by type and tile (VT_*, TILE_*).
typedef void (*GKernel)(GGemm, GEpi);
struct GActKernels {
  GKernel up[3][3], dh[2][4];
};

// h = phi(X Wg^T) * (X Wu^T): A = Wg, A1 = Wu (rows alim), B = X; M = 2 Fp
void gated_up(const Launch& L, int type, const GGemm& g, const GEpi& e);
// out = B A^T: A = Wd, B = h; codes: out_type, scaled
void gated_down(const Launch& L, int type, int out_type, const GGemm& g, const GEpi& e);
// the same of up to FEW_X rows, in place at any alignment; "up" keeps codes as
// fp32, its M is F, and of codes hmax has an entry for 16 columns; "down" of up to TWO_X
// bf16 rows reads the second terms that "up" wrote, e.dup rows further down.  (Aligned
// rows of Wd are read by tiles from more than FEW_DOWN rows on.)
constexpr int FEW_X = 64, TWO_X = FEW_X, FEW_DOWN = 16;
// the same of one row, with rows of the matrices longer than ONE_BYTES: h is fp32 (also
// of gated_few_up where h32), and "up" of codes leaves no hmax
constexpr int ONE_BYTES = 2048;
void gated_one_up(const Launch& L, int type, const GGemm& g, const GEpi& e);
void gated_one_down(const Launch& L, int type, int out_type, const GGemm& g, const GEpi& e);
void gated_few_up(const Launch& L, int type, const GGemm& g, const GEpi& e);
void gated_few_down(const Launch& L, int type, int out_type, const GGemm& g, const GEpi& e);
// dh = dY Wd in the tile, from it and what is kept h, dg and du
void gated_dh(const Launch& L, int type, const GGemm& g, const GEpi& e);
// the same by partials of dh (g.splits, e.part)
void gated_dh_split(const Launch& L, int type, const GGemm& g, const GEpi& e);
// The gradients from dg, du and h: dX = dg Wg + du Wu, dWd = dY^T h, and dWg = dg^T X
// with dWu = du^T X, each if its e.out is there; of one tile
struct GGrads {
  GGemm g[3];
  GEpi e[3];
  int first[4];          // workgroups of the products before each (set by the launch)
  // > 0: units have `share` K blocks each of all tiles in a row, of which work[i] are
  // those of the products before i; part: 2 tiles a unit
  int share, work[4];
  float* part;
};
// workgroups of a tile that the card runs at a time
inline int units_of(int tile) { return tile == TILE_BIG ? 256 : 512; }
void gated_grads(const Launch& L, int type, GGrads a);
// out from the partials of products with their e.part: row n + dup joins row n if dup
// (share > 0: as units' shares left them, work K blocks before this product's)
struct GFinish {
  GGemm g;
  GEpi e;
  int dup;
  int share, work;
};
void gated_finish(const Launch& L, int type, int out_type, const GFinish* f, int n);

// Copies of a call's operands with zeros around: rows x cols elements of es
// bytes, ld apart, to prows x pcols ones (times > 1: so often, below each other).
// scale: the source is a checkpoint's codes, with scale bytes lds apart.
struct GPad {
  const void* src;
  const uint8_t* scale;
  long long lds;
  void* dst;
  long long ld;
  int rows, cols, prows, pcols, times;
  int es;
};
constexpr int GPADS = 6;
struct GPads {
  GPad p[GPADS];
  int n;
};
void gated_pad(const Launch& L, const GPads& p);

// checkpoints: rows x cols of the type to codes and scale bytes, and back
void gated_pack(const Launch& L, int type, const void* X, long long ldx, long long rows, int cols,
                int8_t* codes, long long ldc, uint8_t* scale, long long lds);
void gated_unpack(const Launch& L, int type, const int8_t* codes, long long ldc,
                  const uint8_t* scale, long long lds, long long rows, int cols, void* X,
                  long long ldx);

// codes of rows with a scale each: q = round(x / s), s = max |x| / 127; zeros up
// to zcols columns
void gated_codes(const Launch& L, int type, const void* X, long long ldx, long long rows, int cols,
                 int8_t* codes, long long ldc, int zcols, float* scale);
// the same of fp32 rows of whose numbers the largest are among nmax in hmax, ldmax apart
void gated_codes_h(const Launch& L, const float* H, long long ldh, const float* hmax,
                   long long ldmax, int nmax, int rows, int cols, int8_t* codes, long long ldc, int zcols, float* scale);

}  // namespace hfk
