// Internal declarations of the vocabulary kernels: the softmax head over a
// large vocabulary (cross entropy and distillation, with their gradients) and
// the token embedding with its gradient.
#pragma once

#include "hf_internal.h"

namespace hfk {

// Element type of the rows, the matrices and their gradients.
enum VType { VT_F32 = 0, VT_BF16 = 1 };

// K blocks of the GEMMs are whole multiples of this many elements: widths are
// padded to it in packed rows, and vocabulary pieces and row counts in delta.
constexpr int VPAD = 64;
// Rows of packed operands come in whole tiles of this many.
constexpr int VTILE = 256;
// Output tiles of the GEMMs (m x n): 128 x 128, 256 x 256, 128 x 64, 128 x 32.
enum { TILE_SMALL, TILE_BIG, TILE_N64, TILE_N32 };
inline int tile_m(int t) { return t == TILE_BIG ? 256 : 128; }
inline int tile_n(int t) {
  return t == TILE_BIG ? 256 : t == TILE_N64 ? 64 : t == TILE_N32 ? 32 : 128;
}
// Columns of one entry of row statistics: a wave's part of a vocabulary tile.
inline int tile_stat(int t) { return t == TILE_BIG ? 128 : t == TILE_SMALL ? 64 : 32; }
// exp(z - max) is kept in fp16 times this: with the largest at 2^15, terms down
// to 2^-29 of it (20 less in z) have fp16's 11 bits, and those below an absolute
// 2^-40 of it (as they are, 2^-14 and 2^-25: a word 17 below lost its gradient).
constexpr float EXP_SCALE = 32768.0f;
// fp32 logits of tiles but the largest are summed so many columns at a time, and
// then these sums: 128 + D / 128 additions reach one, not D (2 rows, 1,974 x 1,971:
// dW off by 1.3e-6 in one chain, 4e-7; 130 to 1,024 rows, 50,000 x 768: a loss
// takes 2 to 3% more).  Tiles of 256 x 256 have no registers left for it.
constexpr int SUM_COLS = 128;
inline bool sums_parts(int type, int tile) { return type == VT_F32 && tile != TILE_BIG; }
constexpr int VMAX_SPLITS = 64;
constexpr long long L2_BYTES = 32ll << 20;   // the level-2 caches of the 8 XCDs
constexpr long long L3_BYTES = 256ll << 20;  // the last-level cache

// Device scalars of a call.
struct VocabState {
  int n;           // counted rows
  int err;         // a label, token or id outside the vocabulary was seen
  float gscale;    // tau / denom: factor of both gradients
  double inv;      // 1 / denom
};

// C(m, n) = sum_k A(m, k) B(n, k), stored with m contiguous.
//   A(m, k) = akc ? A[m lda + k] : A[k lda + m],  B likewise.
struct VGemm {
  int M, N, K;
  const void *A, *B;
  long long lda, ldb;
  int alim;        // rows of A that exist: m (akc), or k (not akc)
  int blim;        // rows of B that exist, where they are n
  const VocabState* st;
  const void* X;   // the rows of X (what is packed), if they can be read in
  long long ldx;   // place: used where all T of them count; else null
  int T;
  int dyn;         // 1: N is st->n; 2: K is st->n, rounded up to K blocks
  int splits;      // split-K factor (partials), grid z
  int smax;        // where fewer rows count than N, up to so many (0: no more)
  int tile;
  int thin;        // dW of few rows (TILE_SMALL, splits 1)
};

// The partials of a product whose grid is for gy tiles of rows, of which gya
// have any: the workgroups of the others are given to more splits (a tenth of
// 8,192 rows counted, bf16, 32,000 x 2,048: 649 -> 130 us).  A partial is gya
// tiles of rows; so many of them take no more than splits of gy tiles.
__host__ __device__ inline int splits_of(int splits, int smax, int gy, int gya) {
  const int more = gya > 0 ? splits * gy / gya : splits;
  return smax <= splits ? splits : more < smax ? more : smax;
}

struct VEpi {
  // logits
  float zscale;          // 1 / tau
  float* z;              // logits kept (row n, column m), or null
  void* pt;              // or EXP_SCALE exp(z - max of its statistics entry) in fp16
  long long ldz;
  float2* stat;          // per row and entry: max, sum of exp(z - max)
  int ldstat, tile0;     // entries per row; index of this launch's first
  const int* lab;        // the rows' labels, whose logits go to zt; or null
  float* zt;
  int v0;                // this launch's first column
  const float* lse;      // p: log-sum-exp per row
  void* d;               // delta, row n, column m
  long long ldd;
  // products
  float* part;           // partials, [split][n][m]
  long long ldp;
  int add;               // part += rather than =
  void* out;             // final output, scaled by st->gscale
  long long ldo;
  int accumulate;        // out += rather than =
  int stream;            // (dW of few rows) out past the caches
  const int* idx;        // dX: row of out for a packed row
};

// logits of a vocabulary piece: A = W piece (akc), B = packed rows (akc);
//   stat, and z or pt if kept
void vocab_logits(const Launch& L, int type, const VGemm& g, const VEpi& e);
// p = exp(z - lse) of a vocabulary piece, rounded to the type, into d
void vocab_probs(const Launch& L, int type, const VGemm& g, const VEpi& e);
// row gradients: A = W piece (rows k), B = delta (k contiguous); into part, or,
// with e.out and one split, straight into out
void vocab_dx(const Launch& L, int type, const VGemm& g, const VEpi& e);
// matrix gradient: A = packed rows (rows k), B = delta (rows k); into out, or
// into part where g.splits > 1
void vocab_dw(const Launch& L, int type, const VGemm& g, const VEpi& e);

// -------------------------------------------------------------- row kernels
struct VRows {
  int T;                    // rows of the call
  int V, D, K;              // vocabulary, width, targets per row
  const int32_t* ids;       // T x K targets (labels: K = 1)
  long long ldi;
  const float* t;           // T x K teacher logits, or null (hard labels)
  long long ldt;
  float tau;
  float denom;              // > 0: divides the sum of the losses; 0: counted rows
  VocabState* st;
  int* pos;                 // T: packed row of a row, -1: not counted
  int* idx;                 // the row of a packed row
  int* lab;                 // labels: that of a packed row
  float* row_loss;          // T
};
// which rows count: pos, idx and the state; zero losses for those that do not.
// False: few enough that vocab_pack_rows does it instead.
bool vocab_count(const Launch& L, const VRows& r);
// counted rows of X packed to xp (zeros past the width, and past the last row
// up to a whole tile; twice, dup rows apart, if dup > 0), rows of dX that do
// not count set to zero
// (in_place: not where all rows count; counted: by vocab_count)
void vocab_pack_rows(const Launch& L, int type, const VRows& r, bool counted, const void* X,
                     long long ldx, bool in_place, void* xp, int Dp, int dup, void* dX,
                     long long lddx);
// rows [0, R) of W copied to wp (zeros past the width)
void vocab_pack_matrix(const Launch& L, int type, const void* W, long long ldw,
                       int R, int D, void* wp, int Dp);
struct VTarget {
  float* zt;                // packed row x K: target logits over tau
  int* id;                  // packed row x K: target id, -1: none (or a repeat)
  float* dt;                // packed row x K: delta at the target
};
// log-sum-exp from the statistics, the rows' losses and the targets' delta;
// z: kept logits or null (then a label's is in t.zt, and those of lists are
// formed of X or xp and W).  True: the loss is summed too.
// parts: the logits are summed SUM_COLS at a time.
bool vocab_row_loss(const Launch& L, int type, const VRows& r, bool parts, const float2* stat,
                    int ldstat, int tiles, const float* z, long long ldz, const VTarget& t, float* lse,
                    const void* X, long long ldx, const void* xp, int Dp, const void* W,
                    long long ldw, float* loss);
// loss = sum of the counted rows' losses / denom
void vocab_loss_sum(const Launch& L, const VRows& r, float* loss);
// delta from kept logits of the columns [v0, v0 + Vc), targets included (dup:
// the rounding's rest too, dup rows further down), and the loss unless null.
// z null (bf16): d holds EXP_SCALE exp(z - max) in fp16, by statistics entries of `sg`
// columns.
// self (bf16 with all columns kept): the rows' statistics and losses as well,
// instead of vocab_row_loss; the loss is then still to be summed.
void vocab_delta(const Launch& L, int type, const VRows& r, const float* z, long long ldz,
                 const float2* stat, int tiles, int sg, const float* lse, const VTarget& t,
                 int v0, int Vc, int rows, bool self, void* d, long long ldd, int dup, float* loss);
// delta at the targets within the piece [v0, v0 + Vc)
void vocab_fix(const Launch& L, int type, const VRows& r, const VTarget& t, int v0,
               int Vc, void* d, long long ldd);
// out(row) = gscale (sum over splits, and over the dup copy) part(row) of the
// partials that product g wrote with e; rows: of out, those counted of them
// where counted.  If e.out, nothing where g had one split, which wrote out.
// idx: destination row of a packed row, null: itself; and the loss, unless null
void vocab_finish(const Launch& L, int type, const VGemm& g, const VEpi& e, int dup, int rows,
                  int counted, int D, const int* idx, void* out, long long ldo,
                  int accumulate, const VRows* r, float* loss);

// ---------------------------------------------------------------- embedding
struct VSort {
  int* key;                 // T: ids in order
  int* pos;                 // T: their rows
  int* tkey;                // T: scratch
  int* tpos;
  unsigned* hist;           // histograms of the radix passes
  float* part;              // sums of tokens that reach over a run's ends
};
// unsigned words of hist, and floats of part, for T rows
size_t vocab_sort_hist(long long T, int V);
size_t vocab_sort_part(long long T, int D, int type);
void vocab_embed(const Launch& L, int type, const void* E, long long lde, int V, int D,
                 const int32_t* tok, int T, float scale, void* out, long long ldo,
                 VocabState* st);
void vocab_embed_grad(const Launch& L, int type, const int32_t* tok, int T, int V, int D,
                      float scale, const void* dout, long long ldd, void* dE,
                      long long lde, int accumulate, const VSort& s, VocabState* st);

}  // namespace hfk
