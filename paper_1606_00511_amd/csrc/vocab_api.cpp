// Host side of the vocabulary calls declared in include/hf.h: context,
// argument validation, workspace carve-up and the order of the kernels.
//
// The head works on packed rows (the N that count, N known to the device
// only) in one of two ways, chosen by the call's sizes:
//   kept        the logits of the call fit KEEP_BYTES, in fp32 or (bf16) as
//               exponentials in fp16: computed once, turned into delta
//   recomputed  one pass over the whole vocabulary for the statistics, then
//               piece by piece the logits again, straight into delta, and the
//               piece's share of dX and rows of dW.  The first piece is the
//               pass's last, and its logits are kept: they need no second
//               computation
// A loss without its gradient keeps none, but for few rows with lists, whose
// targets' are then read there.
#include "hf.h"
#include "call_context.h"
#include "gemm_shape.h"
#include "vocab_internal.h"

#include <algorithm>
#include <cmath>
#include <new>

using namespace hfk;

namespace {

constexpr size_t MiB = (size_t)1 << 20;
constexpr size_t KEEP_BYTES = 1536 * MiB;    // kept logits
constexpr size_t WPACK_BYTES = 256 * MiB;    // packed rows of W
constexpr int TWO_TERM_ROWS = 128;

struct Layout {
  size_t state, pos, idx, rloss, lse, zt, tid, tdt, stat, xp, wp, z, partx, partw;
  size_t key, spos, tkey, tpos, hist, epart, need;
};

}  // namespace

struct hf_vocab : hfk::CallContext {
  int V = 0, D = 0, Dp = 0, type = 0, es = 0;
  int64_t Rmax = 0, Rws = 0;
  char* ws = nullptr;
  Layout lay = {};

  template <class T>
  T* at(size_t off) const { return reinterpret_cast<T*>(ws + off); }
  VocabState* st() const { return at<VocabState>(lay.state); }
};

namespace {

// ------------------------------------------------------------------ sizes
inline int64_t tile_rows(int64_t T) { return std::max<int64_t>(up(T, VTILE), VTILE); }

// bf16 calls of at most TWO_TERM_ROWS rows hold delta as two bf16 terms: with
// few rows nothing averages the rounding of the label's entry, and the matrix
// cores wait for W anyway.
inline int two_term(const hf_vocab* c, int64_t T) {
  return c->type == VT_BF16 && T > 0 && T <= TWO_TERM_ROWS ? (int)up(T, VPAD / 2) : 0;
}
// Rows of delta: whole tiles; of few rows, whose logits are kept however many
// they are, no more than the K blocks of dW's product read.
inline int64_t delta_rows(const hf_vocab* c, int64_t T) {
  if (T > TWO_TERM_ROWS) return tile_rows(T);
  const int dup = two_term(c, T);
  return dup ? 2 * dup : up(T, VPAD);
}
// Bytes of a column of what is kept and of delta, which takes its place; few
// bf16 rows keep fp32 logits beside delta.
inline size_t col_bytes(const hf_vocab* c, int64_t T) {
  return (size_t)delta_rows(c, T) * c->es + (two_term(c, T) ? (size_t)T * 4 : 0);
}
inline bool keeps(const hf_vocab* c, int64_t T) {
  return T <= TWO_TERM_ROWS || col_bytes(c, T) * up(c->V, VTILE) <= KEEP_BYTES;
}
// Whether a loss alone with lists of K targets keeps its logits, in fp32, to read
// the targets' there, rather than form these again (vocab_tlogit: a launch, rows
// of W at 7 TB/s, and a wave waits about 1 us for memory every 64 (fp32) or 128
// columns); us either way
inline bool reads_lists(const hf_vocab* c, int64_t T, int K) {
  if (T > TWO_TERM_ROWS && (c->type != VT_F32 || !keeps(c, T))) return false;
  const double keep = 4.0 * (double)T * c->V / 6e6;
  const double again = 4.0 + c->D / (c->type == VT_F32 ? 64.0 : 128.0) +
                       (double)T * K * c->D * c->es / 7e6;
  return keep < again;
}
// columns of a piece: as many as are kept
inline int piece_cols(const hf_vocab* c, int64_t T) {
  return (int)std::max<int64_t>((int64_t)(KEEP_BYTES / col_bytes(c, T)) / 1024 * 1024, 1024);
}
// rows of W packed at a time
inline int pack_rows(const hf_vocab* c) {
  const int64_t n = (int64_t)(WPACK_BYTES / ((size_t)c->Dp * c->es)) / 1024 * 1024;
  return (int)std::min<int64_t>(c->V, std::max<int64_t>(n, 1024));
}
inline size_t z_bytes(const hf_vocab* c, int64_t T) {
  return col_bytes(c, T) * (keeps(c, T) ? up(c->V, VTILE) : piece_cols(c, T));
}

void plan(const hf_vocab* c, int64_t R, Layout* l) {
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t o = off;
    off += (bytes + 255) & ~size_t(255);
    return o;
  };
  const size_t r = (size_t)R, Rp = (size_t)tile_rows(R);
  l->state = take(sizeof(VocabState));
  l->pos = take(r * 4);
  l->idx = take(r * 4);
  l->rloss = take(r * 4);
  l->lse = take(Rp * 4);
  l->zt = take(r * HF_VOCAB_MAX_TOP * 4);
  l->tid = take(r * HF_VOCAB_MAX_TOP * 4);
  l->tdt = take(r * HF_VOCAB_MAX_TOP * 4);
  // (few rows: entries of 32 columns, else of 64 or 128)
  l->stat = take(std::max(std::min<size_t>(r, FEW_ROWS) * (size_t)(c->V / 32 + 8),
                          r * (size_t)(c->V / 64 + 8)) * sizeof(float2));
  l->xp = take(Rp * c->Dp * c->es);
  l->wp = take((size_t)pack_rows(c) * c->Dp * c->es);
  // what the largest of up to R rows needs: few rows, kept logits, pieces
  size_t zb = z_bytes(c, std::min<int64_t>(R, TWO_TERM_ROWS));
  if (R > TWO_TERM_ROWS)
    zb = std::max(zb, keeps(c, R) ? z_bytes(c, R) : KEEP_BYTES);
  l->z = take(zb);
  l->partx = take(std::max(Rp * (size_t)c->Dp, SPLIT_FLOATS) * 4);
  l->partw = take(SPLIT_FLOATS * 4);
  l->key = take(r * 4);
  l->spos = take(r * 4);
  l->tkey = take(r * 4);
  l->tpos = take(r * 4);
  l->hist = take(vocab_sort_hist(R, c->V) * 4);
  l->epart = take(vocab_sort_part(R, c->D, c->type) * 4);
  l->need = off;
}
size_t plan_bytes(const hf_vocab* c, int64_t R) {
  Layout l;
  plan(c, R, &l);
  return l.need;
}

// ----------------------------------------------------------------- checks
// (arguments first, then whether the workspace serves the rows)
int check_rows(hf_vocab* c, int64_t T) {
  if (T < 0 || T > c->Rmax)
    return fail(c, HF_EINVAL, "%lld rows outside [0, %lld]", (long long)T, (long long)c->Rmax);
  return HF_OK;
}
int check_ready(hf_vocab* c, int64_t T) {
  if (!c->ws) return fail(c, HF_EWORKSPACE, "no workspace set (hf_vocab_set_workspace)");
  if (T > c->Rws)
    return fail(c, HF_EWORKSPACE, "%lld rows above the %lld the workspace serves", (long long)T,
                (long long)c->Rws);
  return HF_OK;
}
// -------------------------------------------------------------- the passes
int end(hf_vocab* c) {
  HIP_TRY(c, hipGetLastError());
  return HF_OK;
}

struct Grad {
  void* dX;
  int64_t lddx;
  void* dW;
  int64_t lddw;
  int accumulate;
};

void head(hf_vocab* c, VRows r, const void* X, int64_t ldx, const void* W, int64_t ldw,
          float* loss, const Grad* g) {
  const Launch L{c->stream, nullptr};
  const Layout& l = c->lay;
  const int T = r.T, V = c->V, D = c->D, Dp = c->Dp, type = c->type, es = c->es;
  r.V = V;
  r.D = D;
  r.st = c->st();
  r.pos = c->at<int>(l.pos);
  r.idx = c->at<int>(l.idx);
  r.lab = c->at<int>(l.tid);
  if (!r.row_loss) r.row_loss = c->at<float>(l.rloss);
  const bool keep = g && keeps(c, T);
  const bool lists = !g && r.t && reads_lists(c, T, r.K);
  const int dup = keep ? two_term(c, T) : 0;
  float* lse = c->at<float>(l.lse);
  float2* stat = c->at<float2>(l.stat);
  void* xp = c->at<void>(l.xp);

  // rows of X that the GEMMs can read in place are not packed if all of them
  // count (which the device finds out)
  const bool in_place = !dup && D % VPAD == 0 && ldx <= MAX_LD && (uintptr_t)X % 16 == 0 &&
                        (ldx * es) % 16 == 0;
  const void* xd = in_place ? X : nullptr;
  const bool counted = vocab_count(L, r);
  vocab_pack_rows(L, type, r, counted, X, ldx, in_place, xp, Dp, dup, g ? g->dX : nullptr,
                  g ? g->lddx : 0);

  // W as it is where the GEMMs' 16-byte loads can read it, else packed, at
  // most pack_rows at a time
  const bool direct = D % VPAD == 0 && ldw <= MAX_LD && (uintptr_t)W % 16 == 0 &&
                      (ldw * es) % 16 == 0;
  const int wrows = direct ? V : pack_rows(c);
  int packed = -1, packed_n = 0;        // the packed piece
  auto matrix = [&](int v0, int n, long long* ld) -> const void* {
    if (direct) {
      *ld = ldw;
      return (const char*)W + (size_t)v0 * ldw * es;
    }
    void* wp = c->at<void>(l.wp);
    if (packed != v0 || packed_n < n)
      vocab_pack_matrix(L, type, (const char*)W + (size_t)v0 * ldw * es, ldw, n, D, wp, Dp);
    packed = v0;
    packed_n = n;
    *ld = Dp;
    return wp;
  };

  // ---- statistics of the whole vocabulary, and the logits of the first piece
  // (with `keep`, all of them)
  const int Rp = (int)tile_rows(T);
  const int vc = !g || keep ? V : piece_cols(c, T);
  const long long ldd = up(vc, VTILE);
  // fp32: logits, then delta in their place; bf16: exponentials, then delta;
  // few bf16 rows: fp32 logits, and delta behind them
  const bool f16 = type == VT_BF16 && !dup && !lists;
  float* z = (g && !f16) || lists ? c->at<float>(l.z) : nullptr;
  void* d = !g ? nullptr : dup ? (void*)(z + (size_t)T * ldd) : c->at<void>(l.z);
  const int sstep = std::min(wrows, vc);
  const int tile = shape_for(type, sstep, T, Dp, false, g && f16 ? 2 : 4).tile;
  const int sg = tile_stat(tile);
  const int tiles = (V + sg - 1) / sg;
  VEpi e = {};
  e.zscale = 1.0f / r.tau;
  e.stat = stat;
  e.ldstat = tiles;
  // labels' logits that are not kept in fp32
  const bool dots = (!keep && !lists) || f16;
  VTarget tg = {c->at<float>(l.zt), nullptr, nullptr};
  if (dots && !r.t) {
    e.lab = r.lab;
    e.zt = tg.zt;
  }
  auto logits = [&](int v0, int n, bool keep_it) {
    VGemm q = {};
    q.A = matrix(v0, n, &q.lda);
    q.B = xp;
    q.ldb = Dp;
    q.M = n;
    q.N = T;
    q.K = Dp;
    q.alim = n;
    q.blim = Rp;
    q.st = r.st;
    q.X = xd;
    q.ldx = ldx;
    q.T = T;
    q.dyn = 1;
    q.splits = 1;
    q.tile = tile;
    e.tile0 = v0 / sg;
    e.v0 = v0;
    e.z = keep_it && z ? z + v0 : nullptr;
    e.pt = keep_it && f16 ? (char*)d + (size_t)v0 * 2 : nullptr;
    e.ldz = ldd;
    vocab_logits(L, type, q, e);
  };
  const int kept = g || lists ? std::min(vc, V) : 0;
  for (int v0 = kept; v0 < V; v0 += wrows) logits(v0, std::min(wrows, V - v0), false);
  for (int v0 = 0; v0 < kept; v0 += wrows) logits(v0, std::min(wrows, kept - v0), true);

  // ---- losses
  if (g) {
    tg.id = c->at<int>(l.tid);
    tg.dt = c->at<float>(l.tdt);
  }
  const bool self = dup > 0;             // few rows: with delta
  bool summed = false;
  if (!self)
    summed = vocab_row_loss(L, type, r, sums_parts(type, tile), stat, tiles, tiles,
                            dots ? nullptr : z, ldd, tg, lse, xd, ldx, xp, Dp, W, ldw, loss);
  if (g && T > 0)
    vocab_delta(L, type, r, z, ldd, stat, tiles, sg, lse, tg, 0, std::min(vc, V),
                dup ? dup : (int)up(T, VPAD), self, d, ldd, dup, self || summed ? nullptr : loss);
  if (!summed && (!g || T < 1 || (self && !g->dX))) vocab_loss_sum(L, r, loss);
  if (!g) return;

  // ---- gradients, piece by piece
  // rows of dX's products: the counted ones, or both terms of few
  const int xrows = dup ? 2 * dup : T;
  float* partx = c->at<float>(l.partx);
  Shape xs = {0, 1};
  VGemm xq = {};
  VEpi xe = {};
  int xmax = 0;
  for (int p0 = 0; p0 < V; p0 += vc) {
    const int pn = std::min(vc, V - p0);
    // a piece of delta covers several packed pieces of W where logits are kept
    for (int v0 = p0; v0 < p0 + pn; v0 += wrows) {
      const int n = std::min(wrows, p0 + pn - v0);
      long long lda = 0;
      const void* A = nullptr;
      if (p0 > 0 || g->dX) A = matrix(v0, n, &lda);
      char* dv = (char*)d + (size_t)(v0 - p0) * es;
      if (p0 > 0) {
        VGemm q = {};
        q.A = A;
        q.lda = lda;
        q.B = xp;
        q.ldb = Dp;
        q.M = n;
        q.N = T;
        q.K = Dp;
        q.alim = n;
        q.blim = Rp;
        q.st = r.st;
        q.X = xd;
        q.ldx = ldx;
        q.T = T;
        q.dyn = 1;
        q.splits = 1;
        q.tile = shape_for(type, n, T, Dp, false, 2).tile;
        VEpi pe = {};
        pe.zscale = 1.0f / r.tau;
        pe.lse = lse;
        pe.d = dv;
        pe.ldd = ldd;
        vocab_probs(L, type, q, pe);
        vocab_fix(L, type, r, tg, v0, n, dv, ldd);
      }
      if (!g->dX || T < 1) continue;
      VGemm q = {};
      q.A = A;
      q.lda = lda;
      q.B = dv;
      q.ldb = ldd;
      q.M = D;
      q.N = xrows;
      q.K = n;
      q.alim = n;
      q.blim = (int)delta_rows(c, T);
      q.st = r.st;
      q.dyn = dup ? 0 : 1;
      if (v0 == 0) {
        xs = shape_for(type, D, xrows, n, true, 4);
        xmax = (int)std::min<int64_t>(VMAX_SPLITS, n / 256);
        xe.part = partx;
        xe.ldp = Dp;
        // one piece and no splits: straight into dX
        if (n == V && xs.splits == 1 && !dup && xs.tile < TILE_N64) {
          xe.out = g->dX;
          xe.ldo = g->lddx;
          xe.idx = r.idx;
        }
      }
      q.splits = xs.splits;
      q.smax = xmax;
      q.tile = xs.tile;
      xe.add = v0 > 0;
      vocab_dx(L, type, q, xe);
      xq = q;
    }
    if (!g->dW) continue;
    VGemm q = {};
    q.A = xp;
    q.lda = Dp;
    q.ldb = ldd;
    q.M = D;
    q.K = dup ? 2 * dup : (int)up(T, VPAD);
    q.alim = dup ? 2 * dup : Rp;
    q.st = r.st;
    q.dyn = dup ? 0 : 2;
    q.X = xd;
    q.ldx = ldx;
    q.T = T;
    q.thin = q.K <= (type == VT_F32 ? 64 : 256) && (int64_t)pn * D >= (1 << 20);
    Shape ws = {TILE_SMALL, 1, 0.0}, rest = ws;
    int n1 = pn;
    if (!q.thin) {
      ws = shape_for(type, D, pn, q.K, true, 2);
      // a last round of few tiles leaves most units idle: its rows of dW are a
      // product of their own then, of a shape of their own (788 tiles of 256, K
      // = 2,251: 310 -> 282 us)
      double least = ws.us;
      for (int tile : {TILE_BIG, TILE_SMALL}) {
        const int64_t rn = tile_n(tile), tm = (D + tile_m(tile) - 1) / tile_m(tile);
        const int64_t slots = tile == TILE_BIG ? 256 : 512;
        const int64_t whole = tm * ((pn + rn - 1) / rn) / slots * slots / tm * rn;
        if (whole <= 0 || whole >= pn) continue;
        const Shape a = shape_for(type, D, whole, q.K, true, 2);
        const Shape b = shape_for(type, D, pn - whole, q.K, true, 2);
        if (a.us + b.us + 4.0 < least) {
          least = a.us + b.us + 4.0;
          ws = a;
          rest = b;
          n1 = (int)whole;
        }
      }
    }
    auto product = [&](int r0, int n, const Shape& h) {
      q.B = (const char*)d + (size_t)r0 * es;
      q.N = n;
      q.tile = h.tile;
      q.splits = h.splits;
      VEpi pe = {};
      char* out = (char*)g->dW + (size_t)(p0 + r0) * g->lddw * es;
      pe.part = c->at<float>(l.partw);
      pe.ldp = Dp;
      pe.out = out;
      pe.ldo = g->lddw;
      pe.accumulate = g->accumulate;
      // (rows that share lines go through the caches: 118,135 x 4,068 of fp32 took
      // 2,917 us, past them 3,087)
      pe.stream = (long long)V * D * es > L2_BYTES && (uintptr_t)out % 128 == 0 &&
                  (g->lddw * es) % 128 == 0;
      vocab_dw(L, type, q, pe);
      if (q.splits > 1)
        vocab_finish(L, type, q, pe, 0, n, 0, D, nullptr, out, g->lddw, g->accumulate, nullptr,
                     nullptr);
    };
    product(0, n1, ws);
    if (n1 < pn) product(n1, pn - n1, rest);
  }
  if (g->dX && T > 0)
    vocab_finish(L, type, xq, xe, dup, T, 1, D, r.idx, g->dX, g->lddx, 0, &r,
                 self ? loss : nullptr);
}

// arguments of a head call, then its work
int head_call(hf_vocab* c, const void* X, int64_t ldx, const void* W, int64_t ldw,
              const int32_t* ids, int64_t ldi, const float* t, int64_t ldt, int32_t K, float tau,
              int64_t T, float denom, float* loss, float* row_loss, const Grad* g,
              const char* ids_name) {
  int rc;
  if (!c) return HF_EINVAL;
  if ((rc = check_rows(c, T)) ||
      (rc = check_mat(c, X, ldx, c->D, c->es, T, "X")) ||
      (rc = check_mat(c, W, ldw, c->D, c->es, c->V, "W")) ||
      (rc = check_mat(c, ids, ldi, K, 4, T, ids_name)) ||
      (t && (rc = check_mat(c, t, ldt, K, 4, T, "t"))) ||
      (rc = check_mat(c, loss, 1, 1, 4, 1, "loss")) ||
      (row_loss && (rc = check_mat(c, row_loss, 1, 1, 4, T, "row_loss"))))
    return rc;
  if (!(denom >= 0.0f) || std::isinf(denom))
    return fail(c, HF_EINVAL, "denom %g is not a finite number >= 0", (double)denom);
  if (g) {
    if (!g->dX && !g->dW) return fail(c, HF_EINVAL, "neither dX nor dW given");
    if ((g->dX && (rc = check_mat(c, g->dX, g->lddx, c->D, c->es, T, "dX"))) ||
        (g->dW && (rc = check_mat(c, g->dW, g->lddw, c->D, c->es, c->V, "dW"))))
      return rc;
    if ((rc = check_apart(c, X, "X", g->dX, "dX", T)) ||
        (rc = check_apart(c, W, "W", g->dW, "dW", 1)))
      return rc;
    if (g->accumulate != 0 && g->accumulate != 1)
      return fail(c, HF_EINVAL, "accumulate %d is neither 0 nor 1", g->accumulate);
  }
  if ((rc = check_ready(c, T)) || (rc = follow(c, true))) return rc;
  VRows r = {};
  r.T = (int)T;
  r.K = K;
  r.ids = ids;
  r.ldi = ldi;
  r.t = t;
  r.ldt = ldt;
  r.tau = tau;
  r.denom = denom;
  r.row_loss = row_loss;
  head(c, r, X, ldx, W, ldw, loss, g);
  return end(c);
}

int check_list(hf_vocab* c, const float* t, int64_t T, int32_t K, float tau) {
  if (!c) return HF_EINVAL;
  if (T > 0 && !t) return fail(c, HF_EINVAL, "t is NULL");
  if (K < 1 || K > HF_VOCAB_MAX_TOP)
    return fail(c, HF_EINVAL, "%d teacher logits per row outside [1, %d]", K, HF_VOCAB_MAX_TOP);
  // 1 / tau and tau^2 stay finite and normal
  if (!(tau >= 1e-4f && tau <= 1e4f))
    return fail(c, HF_EINVAL, "tau %g outside [1e-4, 1e4]", (double)tau);
  return HF_OK;
}

}  // namespace

// ==================================================================== C ABI
extern "C" {

int hf_vocab_create(int64_t vocab, int32_t width, int32_t type, int64_t max_rows,
                    void* hip_stream, hf_vocab** out) {
  if (!out) return HF_EINVAL;
  *out = nullptr;
  if (vocab < 1 || vocab > HF_VOCAB_MAX || width < 1 || width > HF_VOCAB_MAX_WIDTH ||
      (type != HF_TYPE_FP32 && type != HF_TYPE_BF16) || max_rows < 1 ||
      max_rows > HF_VOCAB_MAX_ROWS)
    return HF_EINVAL;
  hf_vocab* c = new (std::nothrow) hf_vocab();
  if (!c) return HF_ENOMEM;
  c->V = (int)vocab;
  c->D = width;
  c->Dp = (int)up(width, VPAD);
  c->type = type;
  c->es = type == HF_TYPE_FP32 ? 4 : 2;
  c->Rmax = max_rows;
  c->stream = reinterpret_cast<hipStream_t>(hip_stream);
  *out = c;
  return HF_OK;
}

int hf_vocab_destroy(hf_vocab* c) {
  if (!c) return HF_OK;
  if (c->last) (void)hipEventDestroy(c->last);
  delete c;
  return HF_OK;
}

int hf_vocab_set_stream(hf_vocab* c, void* s) {
  if (!c) return HF_EINVAL;
  c->stream = reinterpret_cast<hipStream_t>(s);
  return c->pending ? follow(c, false) : HF_OK;
}

size_t hf_vocab_workspace_bytes(const hf_vocab* c, int64_t rows) {
  if (!c) return 0;
  if (rows <= 0) rows = c->Rmax;
  if (rows > c->Rmax) return 0;
  return plan_bytes(c, rows);
}

int hf_vocab_set_workspace(hf_vocab* c, void* p, size_t bytes) {
  if (!c) return HF_EINVAL;
  if (!p) return fail(c, HF_EINVAL, "workspace pointer is NULL");
  if ((uintptr_t)p & 255u) return fail(c, HF_EINVAL, "workspace is not 256-byte aligned");
  const size_t need1 = plan_bytes(c, 1);
  if (bytes < need1)
    return fail(c, HF_EWORKSPACE, "workspace of %zu bytes is smaller than the %zu needed "
                "for one row", bytes, need1);
  // the largest number of rows whose layout fits (it grows with the rows)
  int64_t lo = 1, hi = c->Rmax;
  while (lo < hi) {
    const int64_t mid = lo + (hi - lo + 1) / 2;
    if (plan_bytes(c, mid) <= bytes) lo = mid;
    else hi = mid - 1;
  }
  c->ws = nullptr;
  plan(c, lo, &c->lay);
  c->Rws = lo;
  c->pending = false;
  HIP_TRY(c, hipMemset((char*)p + c->lay.state, 0, sizeof(VocabState)));
  HIP_TRY(c, hipDeviceSynchronize());
  c->ws = reinterpret_cast<char*>(p);
  return HF_OK;
}

int hf_vocab_loss(hf_vocab* c, const void* X, int64_t ldx, const void* W, int64_t ldw,
                  const int32_t* y, int64_t rows, float denom, float* loss, float* row_loss) {
  return head_call(c, X, ldx, W, ldw, y, 1, nullptr, 0, 1, 1.0f, rows, denom, loss, row_loss,
                   nullptr, "y");
}

int hf_vocab_loss_grad(hf_vocab* c, const void* X, int64_t ldx, const void* W, int64_t ldw,
                       const int32_t* y, int64_t rows, float denom, float* loss, float* row_loss,
                       void* dX, int64_t lddx, void* dW, int64_t lddw, int32_t accumulate) {
  const Grad g = {dX, lddx, dW, lddw, accumulate};
  return head_call(c, X, ldx, W, ldw, y, 1, nullptr, 0, 1, 1.0f, rows, denom, loss, row_loss, &g,
                   "y");
}

int hf_vocab_distill(hf_vocab* c, const void* X, int64_t ldx, const void* W, int64_t ldw,
                     const int32_t* ids, int64_t ldi, const float* t, int64_t ldt, int32_t top,
                     float tau, int64_t rows, float denom, float* loss, float* row_loss) {
  const int rc = check_list(c, t, rows, top, tau);
  if (rc) return rc;
  return head_call(c, X, ldx, W, ldw, ids, ldi, t, ldt, top, tau, rows, denom, loss, row_loss,
                   nullptr, "ids");
}

int hf_vocab_distill_grad(hf_vocab* c, const void* X, int64_t ldx, const void* W, int64_t ldw,
                          const int32_t* ids, int64_t ldi, const float* t, int64_t ldt,
                          int32_t top, float tau, int64_t rows, float denom, float* loss,
                          float* row_loss, void* dX, int64_t lddx, void* dW, int64_t lddw,
                          int32_t accumulate) {
  const int rc = check_list(c, t, rows, top, tau);
  if (rc) return rc;
  const Grad g = {dX, lddx, dW, lddw, accumulate};
  return head_call(c, X, ldx, W, ldw, ids, ldi, t, ldt, top, tau, rows, denom, loss, row_loss,
                   &g, "ids");
}

int hf_vocab_embed(hf_vocab* c, const void* E, int64_t lde, const int32_t* tok, int64_t rows,
                   float scale, void* out, int64_t ldo) {
  int rc;
  if (!c) return HF_EINVAL;
  if ((rc = check_rows(c, rows)) ||
      (rc = check_mat(c, E, lde, c->D, c->es, c->V, "E")) ||
      (rc = check_mat(c, tok, 1, 1, 4, rows, "tok")) ||
      (rc = check_mat(c, out, ldo, c->D, c->es, rows, "out")) ||
      (rc = check_apart(c, E, "E", out, "out", rows)))
    return rc;
  if (!std::isfinite(scale)) return fail(c, HF_EINVAL, "scale is not finite");
  if ((rc = check_ready(c, rows)) || (rc = follow(c, true))) return rc;
  const Launch L{c->stream, nullptr};
  vocab_embed(L, c->type, E, lde, c->V, c->D, tok, (int)rows, scale, out, ldo, c->st());
  return end(c);
}

int hf_vocab_embed_grad(hf_vocab* c, const int32_t* tok, int64_t rows, float scale,
                        const void* dout, int64_t ldd, void* dE, int64_t lde,
                        int32_t accumulate) {
  int rc;
  if (!c) return HF_EINVAL;
  if ((rc = check_rows(c, rows)) ||
      (rc = check_mat(c, tok, 1, 1, 4, rows, "tok")) ||
      (rc = check_mat(c, dout, ldd, c->D, c->es, rows, "dout")) ||
      (rc = check_mat(c, dE, lde, c->D, c->es, c->V, "dE")) ||
      (rc = check_apart(c, dout, "dout", dE, "dE", rows)))
    return rc;
  if (!std::isfinite(scale)) return fail(c, HF_EINVAL, "scale is not finite");
  if (accumulate != 0 && accumulate != 1)
    return fail(c, HF_EINVAL, "accumulate %d is neither 0 nor 1", accumulate);
  if ((rc = check_ready(c, rows)) || (rc = follow(c, true))) return rc;
  const Launch L{c->stream, nullptr};
  const Layout& l = c->lay;
  const VSort s = {c->at<int>(l.key), c->at<int>(l.spos), c->at<int>(l.tkey), c->at<int>(l.tpos),
                   c->at<unsigned>(l.hist), c->at<float>(l.epart)};
  vocab_embed_grad(L, c->type, tok, (int)rows, c->V, c->D, scale, dout, ldd, dE, lde, accumulate,
                   s, c->st());
  return end(c);
}

int hf_vocab_check(hf_vocab* c) {
  if (!c) return HF_EINVAL;
  if (!c->ws) return HF_OK;
  if (c->pending && c->work != c->stream) HIP_TRY(c, hipStreamSynchronize(c->work));
  HIP_TRY(c, hipStreamSynchronize(c->stream));
  int flag = 0;
  HIP_TRY(c, hipMemcpy(&flag, &c->st()->err, sizeof flag, hipMemcpyDeviceToHost));
  if (flag) {
    const int zero = 0;
    HIP_TRY(c, hipMemcpy(&c->st()->err, &zero, sizeof zero, hipMemcpyHostToDevice));
    return fail(c, HF_ELABEL, "a label, token or id outside [0, %d) was seen", c->V);
  }
  return HF_OK;
}

const char* hf_vocab_last_error(const hf_vocab* c) {
  return c ? c->err.c_str() : "null context";
}

}  // extern "C"
