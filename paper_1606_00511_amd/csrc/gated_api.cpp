// Host side of the gated feed-forward calls declared in include/hf.h: context,
// argument validation, workspace carve-up and the order of the kernels.
//
// Inside, the width and the hidden width are whole multiples of 64 (codes: 128):
// operands that are not, or whose rows the GEMMs' 16-byte loads cannot read, are
// copied to the workspace with zeros around them first.
#include "hf.h"
#include "call_context.h"
#include "gated_internal.h"
#include "gemm_shape.h"

#include <algorithm>
#include <climits>
#include <new>

using namespace hfk;

namespace {

// bf16 calls of at most so many rows hold h, and in the gradient dg and du, as two bf16
// terms, the second what the first's rounding left: h's is half of what Y is off by (2-norm
// 0.0023 with it, 0.0017 without), and up to here the matrix cores wait for the matrices
// anyway.
constexpr int TWO_TERM_ROWS = 128;
constexpr size_t WPACK_BYTES = (size_t)64 << 20;   // packed channels of a product of codes

// Elements (bytes, of codes) between the rows of h, dg and du and of codes, past
// their widths: with rows a power of two apart the 16 rows of a load, and the
// loads of all workgroups, fall on one channel of the caches.
constexpr int LD_GAP = 64, LD_GAP_CODES = 128;

struct Layout {
  size_t part, wg, wu, wd;                    // every call
  size_t xp, yp, xt, yt, h, dgu, gu;          // forward, gradient
  size_t xq, sx, hf, hmax, hq, sh;            // codes
  size_t aq, bq;                              // products of codes
  size_t need;
};

}  // namespace

struct hf_gated : hfk::CallContext {
  int D = 0, F = 0, Dp = 0, Fp = 0, Dc = 0, Fc = 0, act = 0, type = 0, es = 0;
  int64_t Rmax = 0, Rws = 0;
  char* ws = nullptr;
  Layout lay = {};

  template <class T>
  T* at(size_t off) const { return reinterpret_cast<T*>(ws + off); }
  // of split products: of the three gradients' up to 8 splits
  size_t part_floats(int64_t R) const {
    const size_t out = (size_t)up(R, VTILE) * Dp + (size_t)up(Dp, VTILE) * Fp +
                       (size_t)up(2 * Fp, VTILE) * Dp;
    return std::max(SPLIT_FLOATS, std::min(8 * out, 2 * SPLIT_FLOATS));
  }
  size_t ldh() const { return Fp + LD_GAP; }
  size_t ldgu() const { return 2 * Fp + LD_GAP; }
  size_t ldxq() const { return Dc + LD_GAP_CODES; }
  size_t ldhq() const { return Fc + LD_GAP_CODES; }
};

namespace {

// whether a call of T rows has second terms
inline bool two_term(const hf_gated* c, int64_t T) {
  return c->type == VT_BF16 && T > 0 && T <= TWO_TERM_ROWS;
}

void plan(const hf_gated* c, int64_t R, Layout* l) {
  size_t off = 0, need = 0;
  auto take = [&](size_t bytes) {
    const size_t o = off;
    off += (bytes + 255) & ~size_t(255);
    need = std::max(need, off);
    return o;
  };
  const size_t Dp = c->Dp, Fp = c->Fp, Dc = c->Dc, Fc = c->Fc, es = c->es, r = (size_t)R;
  // rows of h, dg, du and of packed rows: whole K blocks, and of few rows both terms
  const size_t rk = (size_t)std::max(up(R, 64), 2 * up(std::min<int64_t>(R, TWO_TERM_ROWS), 64));
  l->part = take(c->part_floats(R) * 4);
  // (as codes: a byte an element, up to 128)
  const size_t wbytes = std::max(Fp * Dp * es, std::max(Fp * Dc, Dp * Fc));
  l->wg = take(wbytes);
  l->wu = take(wbytes);
  l->wd = take(wbytes);
  const size_t start = off;
  l->xp = take(rk * Dp * es);
  l->yp = take(rk * Dp * es);
  l->xt = take(64 * Dp * es);
  l->yt = take(64 * Dp * es);
  l->h = take(rk * c->ldh() * es);
  l->dgu = take(rk * c->ldgu() * es);
  l->gu = take(std::min<size_t>(r, FEW_X) * 2 * Fp * 4);
  off = start;
  l->xq = take(r * c->ldxq());
  l->sx = take(r * 4);
  l->hf = take(r * Fc * 4);
  l->hmax = take(std::max(r * (Fp / 32), std::min<size_t>(r, FEW_X) * (Fp / 16)) * 4);
  l->hq = take(r * c->ldhq());
  l->sh = take(r * 4);
  off = start;
  l->aq = take(r * std::max(Dc, Fc));
  l->bq = take(WPACK_BYTES);
  l->need = need;
}
size_t plan_bytes(const hf_gated* c, int64_t R) {
  Layout l;
  plan(c, R, &l);
  return l.need;
}

// ----------------------------------------------------------------- checks
int check_rows(hf_gated* c, int64_t T) {
  if (T < 0 || T > c->Rmax)
    return fail(c, HF_EINVAL, "%lld rows outside [0, %lld]", (long long)T, (long long)c->Rmax);
  return HF_OK;
}
int check_ready(hf_gated* c, int64_t T) {
  if (!c->ws) return fail(c, HF_EWORKSPACE, "no workspace set (hf_gated_set_workspace)");
  if (T > c->Rws)
    return fail(c, HF_EWORKSPACE, "%lld rows above the %lld the workspace serves", (long long)T,
                (long long)c->Rws);
  return HF_OK;
}
// a rows x cols array on its own
int check_size(hf_gated* c, int64_t rows, int64_t most, int64_t cols) {
  if (rows < 0 || rows > most)
    return fail(c, HF_EINVAL, "%lld rows outside [0, %lld]", (long long)rows, (long long)most);
  if (cols < 1 || cols > HF_GATED_MAX_WIDTH)
    return fail(c, HF_EINVAL, "%lld columns outside [1, %d]", (long long)cols, HF_GATED_MAX_WIDTH);
  return HF_OK;
}
int check_weights(hf_gated* c, const void* Wg, int64_t ldg, const void* Wu, int64_t ldu,
                  const void* Wd, int64_t ldd, int es) {
  int rc;
  if ((rc = check_mat(c, Wg, ldg, c->D, es, c->F, "Wg")) ||
      (rc = check_mat(c, Wu, ldu, c->D, es, c->F, "Wu")) ||
      (rc = check_mat(c, Wd, ldd, c->F, es, c->D, "Wd")))
    return rc;
  return HF_OK;
}
int end(hf_gated* c) {
  HIP_TRY(c, hipGetLastError());
  return HF_OK;
}
inline int blocks_of(int64_t cols) { return (int)((cols + CODE_BLOCK - 1) / CODE_BLOCK); }

// -------------------------------------------------------------- operands
// whether the GEMMs' 16-byte loads can read rows of p where they are
inline bool loads16(const void* p, int64_t ld, int es) {
  return ld <= MAX_LD && (uintptr_t)p % 16 == 0 && ld * es % 16 == 0;
}

// The copies that a call's operands need, made in one launch.
struct Pads {
  GPads all = {};
  // p where it is (in_place), or its copy at dst
  const void* operand(bool in_place, const void* p, int64_t ld, int64_t rows, int cols, int es,
                      void* dst, int64_t prows, int pcols, int times, long long* out_ld) {
    if (in_place) {
      *out_ld = ld;
      return p;
    }
    *out_ld = pcols;
    all.p[all.n++] = GPad{p, nullptr, 0, dst, ld, (int)rows, cols, (int)prows, pcols, times, es};
    return dst;
  }
};

GGemm product(int M, int N, int K) {
  GGemm g = {};
  g.M = M;
  g.N = N;
  g.K = K;
  g.alim = M;
  g.blim = N;
  g.ktail = INT_MAX;
  g.splits = 1;
  return g;
}
// operands that are read where they are
void operands(GGemm* g, const void* A, int64_t lda, const void* A1, int64_t lda1, const void* B,
              int64_t ldb) {
  g->A = A;
  g->A1 = A1;
  g->lda = lda;
  g->lda1 = lda1;
  g->B = B;
  g->ldb = ldb;
}
GEpi epilogue(const hf_gated* c, int64_t T) {
  GEpi e = {};
  e.act = c->act;
  e.F = c->F;
  e.Fp = c->Fp;
  e.T = (int)T;
  e.n1 = INT_MAX;
  return e;
}
void set_out(GEpi* e, void* out, int64_t ldo, int64_t rows, int cols) {
  e->out = out;
  e->ldo = ldo;
  e->nout = (int)rows;
  e->mout = cols;
}
// The tile and the splits of K of a product by its estimated time in us:
//   products  RATE (see gemm_shape.h) a unit, of which two of the smaller tiles share
//             one, and C_TILE to fill the LDS and store a tile
//   units     a unit reads UNIT_BYTES a us (measured on 134 MB by 256 workgroups: 5
//             TB/s, and what one alone reads)
//   memory    both operands once
// Partials are written and read again by a launch of its own, few of them in the
// last-level cache.
constexpr double UNIT_BYTES = 5.5e4, C_TILE[4] = {4.0, 6.0, 3.0, 3.0};
inline int es_of(int type) { return type == VT_F32 ? 4 : type == VT_BF16 ? 2 : 1; }
// one tile's time over k columns, `share` to a unit
inline double tile_us(int type, int tile, double k, bool shared) {
  const double rm = tile_m(tile), rn = tile_n(tile);
  return std::max((shared ? 2.0 : tile == TILE_BIG ? 1.0 : 1.4) * rm * rn * k / RATE[type][tile],
                  (shared ? 2.0 : 1.0) * (rm + rn) * k * es_of(type) / UNIT_BYTES) + C_TILE[tile];
}
inline double parts_us(double bytes) {
  return bytes > 0.0 ? 4.0 + bytes / (bytes < 64e6 ? 2 * BYTES_US : BYTES_US) : 0.0;
}
constexpr int SPLITS[] = {1, 2, 3, 4, 5, 6, 8, 10, 12, 16, 20, 24, 32, 48, 64};
// of K a split takes at least so many columns
inline int64_t split_k(int type) { return type == VT_F32 ? 64 : type == VT_BF16 ? 128 : 256; }
// last: the last columns of a product, which tiles of fewer rows spread over more units
// (3,001 rows, up of 1,021 x 2,731, bf16: 17.2 -> 11.0 us; 5,000 rows, 1,500 x 5,000: 24.9
// -> 17.7)
Shape shape_of(int type, int64_t M, int64_t N, int64_t K, bool split, int shapes,
               bool last = false) {
  Shape best = {0, 1, 1e300};
  const double mem = (double)(M + N) * K * es_of(type) / BYTES_US + 4.0;
  for (int tile = 0; tile < (last || N <= FEW_ROWS ? shapes : std::min(shapes, 2)); ++tile) {
    const int64_t RM = tile_m(tile), RN = tile_n(tile), slots = tile == TILE_BIG ? 256 : 512;
    const int64_t tiles = (M + RM - 1) / RM * ((N + RN - 1) / RN);
    for (int s : SPLITS) {
      if (s > 1 && (!split || K / s < split_k(type) ||
                    (size_t)s * up(N, VTILE) * up(M, VPAD) > SPLIT_FLOATS))
        break;
      const double t = (double)((tiles * s + slots - 1) / slots) *
                       tile_us(type, tile, (double)((K + s - 1) / s),
                               tile != TILE_BIG && tiles * s > 256);
      const double us = std::max(t, mem) + (s > 1 ? parts_us(8.0 * s * (double)M * N) : 0.0);
      if (us < best.us) best = {tile, s, us};
    }
  }
  return best;
}
// A product in one launch or two, by their estimated time: a last round of few tiles
// leaves most units idle, and its columns are then a launch of their own, of a shape
// of their own.  run(g) launches columns [g.m0, g.M); shapes: how many of the tiles
// the product has.
template <class Run>
void ranged(GGemm g, int type, bool split, int shapes, Run run) {
  const int64_t M = g.M, N = g.N, K = g.K;
  Shape a = shape_of(type, M, N, K, split, shapes), b = {};
  int64_t m1 = M;
  double least = a.us;
  for (int tile : {TILE_BIG, TILE_SMALL}) {
    const int64_t rm = tile_m(tile), tn = (N + tile_n(tile) - 1) / tile_n(tile);
    const int64_t slots = tile == TILE_BIG ? 256 : 512;
    const int64_t whole = ((M + rm - 1) / rm * tn) / slots * slots / tn * rm;
    if (whole <= 0 || whole >= M) continue;
    const Shape x = shape_of(type, whole, N, K, split, shapes);
    const Shape y = shape_of(type, M - whole, N, K, split, shapes, true);
    if (x.us + y.us + 4.0 < least) {
      least = x.us + y.us + 4.0;
      a = x;
      b = y;
      m1 = whole;
    }
  }
  g.M = (int)m1;
  g.tile = a.tile;
  g.splits = a.splits;
  run(g);
  if (m1 == M) return;
  g.m0 = (int)m1;
  g.M = (int)M;
  g.tile = b.tile;
  g.splits = b.splits;
  run(g);
}
// a product into e's out: straight, or by partials; dup > 0: the rows of second terms
// are dup rows further down and join the first ones'
template <class Kernel>
void summed(hf_gated* c, const Launch& L, int type, int out_type, const GGemm& all, const GEpi& out,
            int dup, int shapes, Kernel kernel) {
  ranged(all, type, true, shapes, [&](const GGemm& g) {
    GEpi e = out;
    if (g.splits > 1 || dup) {
      e.part = c->at<float>(c->lay.part);
      e.ldp = g.M - g.m0;
    }
    kernel(g, e);
    if (!e.part) return;
    const GFinish f = {g, e, dup, 0, 0};
    gated_finish(L, type, out_type, &f, 1);
  });
}

// The gradients' products: one tile for all of them, and splits of K, of about `per`
// columns each, so that the units are done together.  A tile is launched when a unit has room for it, the longest first.
struct Job {
  int64_t M, N, K;
  bool on, joined;       // joined: by partials even if there is one split
};
double makespan(int type, int tile, const Job (&j)[3], int64_t per, size_t room,
                int (&splits)[3]) {
  const int64_t RM = tile_m(tile), RN = tile_n(tile), slots = tile == TILE_BIG ? 256 : 512;
  int64_t n[3] = {}, all = 0;
  double t[3] = {}, part = 0.0, bytes = 0.0;
  size_t floats = 0;
  const int es = es_of(type);
  for (int i = 0; i < 3; ++i) {
    splits[i] = 1;
    if (!j[i].on) continue;
    splits[i] = (int)std::min<int64_t>((j[i].K + per - 1) / per, VMAX_SPLITS);
    n[i] = (j[i].M + RM - 1) / RM * ((j[i].N + RN - 1) / RN) * splits[i];
    t[i] = (double)((j[i].K + splits[i] - 1) / splits[i]);
    all += n[i];
    bytes += (double)es * (j[i].M * j[i].K + j[i].N * j[i].K + j[i].M * j[i].N);
    if (splits[i] > 1 || j[i].joined) {
      part += 8.0 * splits[i] * (double)j[i].M * j[i].N;
      floats += (size_t)splits[i] * up(j[i].N, VTILE) * up(j[i].M, VPAD);
    }
  }
  if (floats > room) return 1e300;
  // the units' times, as a few groups that are equal
  struct Group {
    double at;
    int64_t units;
  } g[16] = {{0.0, slots}};
  int k = 1;
  double end = 0.0;
  for (;;) {
    int i = -1;
    for (int c = 0; c < 3; ++c)
      if (n[c] > 0 && (i < 0 || t[c] > t[i])) i = c;
    if (i < 0) break;
    int f = 0;
    for (int c = 1; c < k; ++c)
      if (g[c].at < g[f].at) f = c;
    // (whole rounds at once while all units are equal)
    const double one = tile_us(type, tile, t[i], tile != TILE_BIG && all > 256);
    const int64_t rounds = k == 1 ? std::max<int64_t>(n[i] / slots, 1) : 1;
    const int64_t take = std::min(n[i], g[f].units * rounds);
    n[i] -= take;
    const int64_t used = std::min(take, g[f].units);
    const double at = g[f].at + one * (double)rounds;
    end = std::max(end, at);
    if (used == g[f].units || k == 16) g[f].at = at;
    else {
      g[f].units -= used;
      g[k++] = {at, used};
    }
  }
  return std::max(end, bytes / BYTES_US + 4.0) + parts_us(part);
}
void grads_shapes(int type, int dup, size_t room, GGrads* a) {
  Job j[3];
  int64_t K = 0;
  for (int i = 0; i < 3; ++i) {
    j[i] = {a->g[i].M, a->g[i].N, a->g[i].K, a->e[i].out != nullptr, i == 0 && dup};
    if (j[i].on) K = std::max(K, j[i].K);
  }
  double best = 1e300;
  for (int tile : {TILE_SMALL, TILE_BIG})
    for (int q : {1, 2, 3, 4, 5, 6, 8, 10, 12, 16, 24, 32}) {
      const int64_t per = up((K + q - 1) / q, 64);
      if (q > 1 && per < split_k(type)) break;
      int splits[3];
      const double us = makespan(type, tile, j, per, room, splits);
      if (us >= best) continue;
      best = us;
      for (int i = 0; i < 3; ++i) {
        a->g[i].tile = tile;
        a->g[i].splits = splits[i];
      }
    }
  // Or by equal shares of all K blocks (hf_gated_shares_f32), where that promises to be
  // quicker by 15%: units are then at work on different K blocks of neighbouring tiles and
  // share little of what they read, and nearly every tile is left in parts.  (4,096 rows,
  // 1,024 x 2,731, fp32: products 1,056 -> 973 us and sums of partials 43 -> 33; where 11%
  // were promised, 16,384 rows, 256 x 512: 201 -> 197, and 6 -> 26; bf16, whose products
  // wait for their reads, 4,096 rows, 1,024 x 2,731: 139 -> 131, and 0 -> 25.)
  if (type != VT_F32) return;
  best /= 1.15;
  for (int tile : {TILE_SMALL, TILE_BIG}) {
    const int64_t RM = tile_m(tile), RN = tile_n(tile), units = units_of(tile), BK = 32;
    int64_t work[4] = {}, tiles = 0;
    for (int i = 0; i < 3; ++i) {
      const int64_t n = j[i].on ? (j[i].M + RM - 1) / RM * ((j[i].N + RN - 1) / RN) : 0;
      tiles += n;
      work[i + 1] = work[i] + n * (j[i].K / BK);
    }
    if (work[3] >= 1 << 30 || (size_t)(2 * units * RM * RN) > room) continue;
    const int64_t share = (work[3] + units - 1) / units;
    if (share < 32 || 16 * share < K / BK) continue;    // (tiles in many parts)
    const double us = tile_us(type, tile, (double)(share * BK), tile != TILE_BIG) +
                      C_TILE[tile] * (double)(tiles / units + 1) +
                      parts_us(8.0 * (double)(std::min(tiles, units) + units) * RM * RN);
    if (us >= best) continue;
    best = us;
    a->share = (int)share;
    for (int i = 0; i < 4; ++i) a->work[i] = (int)work[i];
    for (int i = 0; i < 3; ++i) a->g[i].tile = tile;
  }
}

}  // namespace

// ==================================================================== C ABI
extern "C" {

int hf_gated_create(int32_t width, int32_t hidden, int32_t act, int32_t type, int64_t max_rows,
                    void* hip_stream, hf_gated** out) {
  if (!out) return HF_EINVAL;
  *out = nullptr;
  if (width < 1 || width > HF_GATED_MAX_WIDTH || hidden < 1 || hidden > HF_GATED_MAX_WIDTH ||
      act < HF_SIGMOID || act > HF_GELU_TANH ||
      (type != HF_TYPE_FP32 && type != HF_TYPE_BF16) || max_rows < 1 ||
      max_rows > HF_GATED_MAX_ROWS)
    return HF_EINVAL;
  hf_gated* c = new (std::nothrow) hf_gated();
  if (!c) return HF_ENOMEM;
  c->D = width;
  c->F = hidden;
  c->Dp = (int)up(width, VPAD);
  c->Fp = (int)up(hidden, VPAD);
  c->Dc = (int)up(width, CPAD);
  c->Fc = (int)up(hidden, CPAD);
  c->act = act;
  c->type = type;
  c->es = type == HF_TYPE_FP32 ? 4 : 2;
  c->Rmax = max_rows;
  c->stream = reinterpret_cast<hipStream_t>(hip_stream);
  *out = c;
  return HF_OK;
}

int hf_gated_destroy(hf_gated* c) {
  if (!c) return HF_OK;
  if (c->last) (void)hipEventDestroy(c->last);
  delete c;
  return HF_OK;
}

int hf_gated_set_stream(hf_gated* c, void* s) {
  if (!c) return HF_EINVAL;
  c->stream = reinterpret_cast<hipStream_t>(s);
  return c->pending ? follow(c, false) : HF_OK;
}

size_t hf_gated_workspace_bytes(const hf_gated* c, int64_t rows) {
  if (!c) return 0;
  if (rows <= 0) rows = c->Rmax;
  if (rows > c->Rmax) return 0;
  return plan_bytes(c, rows);
}

int hf_gated_set_workspace(hf_gated* c, void* p, size_t bytes) {
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
  HIP_TRY(c, hipDeviceSynchronize());      // (calls so far may be at work in it)
  plan(c, lo, &c->lay);
  c->Rws = lo;
  c->pending = false;
  c->ws = reinterpret_cast<char*>(p);
  return HF_OK;
}

int hf_gated_forward(hf_gated* c, const void* X, int64_t ldx, const void* Wg, int64_t ldg,
                     const void* Wu, int64_t ldu, const void* Wd, int64_t ldd, int64_t rows,
                     void* Y, int64_t ldy, int32_t keep, void* kept, int64_t ldk, uint8_t* scale,
                     int64_t lds) {
  int rc;
  if (!c) return HF_EINVAL;
  if ((rc = check_rows(c, rows)) ||
      (rc = check_mat(c, X, ldx, c->D, c->es, rows, "X")) ||
      (rc = check_weights(c, Wg, ldg, Wu, ldu, Wd, ldd, c->es)) ||
      (rc = check_mat(c, Y, ldy, c->D, c->es, rows, "Y")) ||
      (rc = check_apart(c, X, "X", Y, "Y", rows)))
    return rc;
  if (keep != HF_KEEP_NONE && keep != HF_KEEP_FULL && keep != HF_KEEP_CODES)
    return fail(c, HF_EINVAL, "keep %d is none of HF_KEEP_*", keep);
  if (keep != HF_KEEP_NONE &&
      ((rc = check_mat(c, kept, ldk, 2 * (int64_t)c->F, keep == HF_KEEP_FULL ? c->es : 1, rows,
                       "kept")) ||
       (rc = check_apart(c, X, "X", kept, "kept", rows)) ||
       (rc = check_apart(c, Y, "Y", kept, "kept", rows))))
    return rc;
  if (keep == HF_KEEP_CODES &&
      (rc = check_mat(c, scale, lds, 2 * blocks_of(c->F), 1, rows, "scale")))
    return rc;
  if ((rc = check_ready(c, rows)) || (rc = follow(c, true))) return rc;
  if (rows == 0) return HF_OK;
  const Launch L{c->stream, nullptr};
  const Layout& l = c->lay;
  const int T = (int)rows, D = c->D, F = c->F, Dp = c->Dp, Fp = c->Fp, es = c->es;
  const int dup = two_term(c, T) ? T : 0;        // (h's second terms: the next T rows)
  // Rows of Wd that tiles cannot read where they are: reading both terms of more than 32
  // rows of h for every 16 of Wd's costs more than copies for tiles where rows are long (48
  // rows, 1,021 x 2,731: 37 us, by copies 30; 2,001 x 5,003: 96, 52; 300 x 900: 16, 20).
  const bool whole = D == Dp && F == Fp && loads16(Wd, ldd, es);
  if (T <= FEW_X && (whole || !dup || T <= 32 || F <= 2048)) {
    GGemm gu = product(F, T, D), gd = product(D, T, F);
    GEpi eu = epilogue(c, T), ed = epilogue(c, T);
    operands(&gu, Wg, ldg, Wu, ldu, X, ldx);
    eu.h = c->at<void>(l.h);
    eu.ldh = c->ldh();
    eu.dup = ed.dup = dup;
    // (of one row h is fp32, unless its rows of Wd are short)
    const bool one = T == 1 && F * es > ONE_BYTES;
    eu.h32 = one;
    if (one) eu.dup = 0;
    eu.keep = keep;
    eu.kept = kept;
    eu.ldk = ldk;
    if (keep == HF_KEEP_CODES) {        // (a workgroup may have half a block of codes)
      eu.kept = c->at<float>(l.gu);
      eu.ldk = 2 * F;
    }
    if (one && D * es > ONE_BYTES) gated_one_up(L, c->type, gu, eu);
    else gated_few_up(L, c->type, gu, eu);
    if (keep == HF_KEEP_CODES) {
      int8_t* k = (int8_t*)kept;
      const int once = F % CODE_BLOCK ? F : 2 * F;     // (no block has both g and u)
      for (int f = 0; f < 2 * F; f += once)
        gated_pack(L, VT_F32, (const float*)eu.kept + f, 2 * F, T, once, k + f, ldk,
                   scale + blocks_of(f), lds);
    }
    set_out(&ed, Y, ldy, T, D);
    if (T > FEW_DOWN && whole) {
      // (each row of h once for 128 of Wd's: 24 rows, 4,096 x 16,384: 45 -> 40 us with
      // the partials)
      gd = product(D, T + dup, F);
      operands(&gd, Wd, ldd, nullptr, 0, eu.h, eu.ldh);
      summed(c, L, c->type, c->type, gd, ed, dup, 4, [&](const GGemm& g, const GEpi& e) {
        gated_down(L, c->type, c->type, g, e);
      });
    } else {
      operands(&gd, Wd, ldd, nullptr, 0, eu.h, eu.ldh);
      if (one) gated_one_down(L, c->type, c->type, gd, ed);
      else gated_few_down(L, c->type, c->type, gd, ed);
    }
    return end(c);
  }
  GGemm gu = product(2 * Fp, T, Dp), gd = product(Dp, T + dup, Fp);
  GEpi eu = epilogue(c, T), ed = epilogue(c, T);
  eu.dup = dup;
  Pads pads;
  gu.B = pads.operand(D == Dp && loads16(X, ldx, es), X, ldx, T, D, es, c->at<void>(l.xp), T, Dp, 1,
                      &gu.ldb);
  const bool pair = D == Dp && ldg == ldu && loads16(Wg, ldg, es) && loads16(Wu, ldu, es);
  gu.A = pads.operand(pair, Wg, ldg, F, D, es, c->at<void>(l.wg), Fp, Dp, 1, &gu.lda);
  gu.A1 = pads.operand(pair, Wu, ldu, F, D, es, c->at<void>(l.wu), Fp, Dp, 1, &gu.lda);
  gu.alim = F;
  gd.A = pads.operand(F == Fp && loads16(Wd, ldd, es), Wd, ldd, D, F, es, c->at<void>(l.wd), D, Fp, 1,
                      &gd.lda);
  gd.alim = D;
  gated_pad(L, pads.all);

  eu.h = c->at<void>(l.h);
  eu.ldh = c->ldh();
  eu.keep = keep;
  eu.kept = kept;
  eu.ldk = ldk;
  eu.ks = scale;
  eu.ldks = lds;
  ranged(gu, c->type, false, 3, [&](const GGemm& g) { gated_up(L, c->type, g, eu); });

  gd.B = eu.h;
  gd.ldb = c->ldh();
  set_out(&ed, Y, ldy, T, D);
  summed(c, L, c->type, c->type, gd, ed, dup, 4, [&](const GGemm& g, const GEpi& e) {
    gated_down(L, c->type, c->type, g, e);
  });
  return end(c);
}

int hf_gated_grad(hf_gated* c, const void* X, int64_t ldx, const uint8_t* xscale, int64_t ldxs,
                  const void* Wg, int64_t ldg, const void* Wu, int64_t ldu, const void* Wd,
                  int64_t ldd, int32_t keep, const void* kept, int64_t ldk, const uint8_t* scale,
                  int64_t lds, const void* dY, int64_t lddy, int64_t rows, void* dX, int64_t lddx,
                  void* dWg, int64_t lddg, void* dWu, int64_t lddu, void* dWd, int64_t lddd,
                  int32_t accumulate) {
  int rc;
  if (!c) return HF_EINVAL;
  if (keep != HF_KEEP_FULL && keep != HF_KEEP_CODES)
    return fail(c, HF_EINVAL, "keep %d is neither HF_KEEP_FULL nor HF_KEEP_CODES", keep);
  if ((rc = check_rows(c, rows)) ||
      (rc = check_mat(c, X, ldx, c->D, xscale ? 1 : c->es, rows, "X")) ||
      (xscale && (rc = check_mat(c, xscale, ldxs, blocks_of(c->D), 1, rows, "xscale"))) ||
      (rc = check_weights(c, Wg, ldg, Wu, ldu, Wd, ldd, c->es)) ||
      (rc = check_mat(c, kept, ldk, 2 * (int64_t)c->F, keep == HF_KEEP_FULL ? c->es : 1, rows,
                      "kept")) ||
      (keep == HF_KEEP_CODES &&
       (rc = check_mat(c, scale, lds, 2 * blocks_of(c->F), 1, rows, "scale"))) ||
      (rc = check_mat(c, dY, lddy, c->D, c->es, rows, "dY")))
    return rc;
  if (!dX && !dWg && !dWu && !dWd) return fail(c, HF_EINVAL, "no gradient given");
  if ((dX && (rc = check_mat(c, dX, lddx, c->D, c->es, rows, "dX"))) ||
      (dWg && (rc = check_mat(c, dWg, lddg, c->D, c->es, c->F, "dWg"))) ||
      (dWu && (rc = check_mat(c, dWu, lddu, c->D, c->es, c->F, "dWu"))) ||
      (dWd && (rc = check_mat(c, dWd, lddd, c->F, c->es, c->D, "dWd"))))
    return rc;
  if ((rc = check_apart(c, X, "X", dX, "dX", rows)) ||
      (rc = check_apart(c, dY, "dY", dX, "dX", rows)) ||
      (rc = check_apart(c, kept, "kept", dX, "dX", rows)) ||
      (rc = check_apart(c, Wg, "Wg", dWg, "dWg", 1)) ||
      (rc = check_apart(c, Wu, "Wu", dWu, "dWu", 1)) ||
      (rc = check_apart(c, Wd, "Wd", dWd, "dWd", 1)) ||
      (rc = check_apart(c, dWg, "dWg", dWu, "dWu", 1)))
    return rc;
  if (accumulate != 0 && accumulate != 1)
    return fail(c, HF_EINVAL, "accumulate %d is neither 0 nor 1", accumulate);
  if ((rc = check_ready(c, rows)) || (rc = follow(c, true))) return rc;
  const Launch L{c->stream, nullptr};
  const Layout& l = c->lay;
  const int T = (int)rows, D = c->D, F = c->F, Dp = c->Dp, Fp = c->Fp, es = c->es, type = c->type;
  const int dup = two_term(c, T) ? (int)up(T, 64) : 0;    // (rows are K: whole K blocks)
  const int Tp = (int)up(T, 64), Kt = dup ? 2 * dup : Tp, T0 = T / 64 * 64;
  GGrads all = {};
  GGemm &gx = all.g[0], &gd = all.g[1], &gw = all.g[2];
  GEpi &ex = all.e[0], &ed = all.e[1], &ew = all.e[2];
  gx = product(Dp, dup ? 2 * dup : T, 2 * Fp);
  gd = product(Fp, Dp, Kt);
  gw = product(Dp, dWg && dWu ? 2 * Fp : Fp, Kt);
  ex = ed = ew = epilogue(c, T);
  ed.accumulate = ew.accumulate = accumulate;
  set_out(&ex, dX, lddx, T, D);
  set_out(&ed, dWd, lddd, D, F);
  set_out(&ew, dWg ? dWg : dWu, dWg ? lddg : lddu, F, D);
  ew.n1 = dWg && dWu ? Fp : INT_MAX;
  ew.out1 = dWu;
  ew.ldo1 = lddu;
  GFinish f[3];
  int n = 0;
  if (T == 0) {
    // the sum of nothing
    for (int i = 1; i < 3 && !accumulate; ++i) {
      all.g[i].splits = 0;
      if (all.e[i].out) f[n++] = {all.g[i], all.e[i], 0, 0, 0};
    }
    gated_finish(L, type, type, f, n);
    return end(c);
  }

  Pads pads;
  const bool weights = D == Dp && F == Fp && ldg == ldu && loads16(Wg, ldg, es) &&
                       loads16(Wu, ldu, es) && loads16(Wd, ldd, es);
  GGemm gh = product(Fp, Tp, Dp);
  gh.A = pads.operand(weights, Wd, ldd, D, F, es, c->at<void>(l.wd), Dp, Fp, 1, &gh.lda);
  if (dX) {
    gx.A = pads.operand(weights, Wg, ldg, F, D, es, c->at<void>(l.wg), Fp, Dp, 1, &gx.lda);
    gx.A1 = pads.operand(weights, Wu, ldu, F, D, es, c->at<void>(l.wu), Fp, Dp, 1, &gx.lda);
  }
  // rows of X and dY: whole K blocks (few bf16 rows: both copies), or where they
  // are, with the last block's in a copy
  const int prows = dup ? dup : Tp, times = dup ? 2 : 1;
  auto rows_of = [&](const void* p, int64_t ld, size_t copy, size_t tail, bool need_k,
                     const void** at, long long* ldat, long long* out_ld) -> const void* {
    const bool place = D == Dp && loads16(p, ld, es) && !(dup && need_k);
    const void* q = pads.operand(place, p, ld, T, D, es, c->at<void>(copy), prows, Dp, times, out_ld);
    if (place && need_k && T % 64)
      *at = pads.operand(false, (const char*)p + (size_t)T0 * ld * es, ld, T - T0, D, es,
                         c->at<void>(tail), 64, Dp, 1, ldat);
    return q;
  };
  gh.B = rows_of(dY, lddy, l.yp, l.yt, dWd != nullptr, &gd.bt, &gd.ldbt, &gh.ldb);
  gh.blim = T;
  gd.B = gh.B;
  gd.ldb = gh.ldb;
  gd.ktail = gw.ktail = T0;
  if (ew.out && xscale) {
    gw.A = pads.operand(false, X, ldx, T, D, es, c->at<void>(l.xp), prows, Dp, times, &gw.lda);
    GPad& p = pads.all.p[pads.all.n - 1];
    p.scale = xscale;
    p.lds = ldxs;
  } else if (ew.out) {
    gw.A = rows_of(X, ldx, l.xp, l.xt, true, &gw.at, &gw.ldat, &gw.lda);
  }
  gated_pad(L, pads.all);

  GEpi eh = epilogue(c, T);
  eh.h = c->at<void>(l.h);
  eh.ldh = c->ldh();
  eh.dgu = c->at<void>(l.dgu);
  eh.lddgu = c->ldgu();
  eh.dup = dup;
  eh.keep = keep;
  eh.kept = const_cast<void*>(kept);
  eh.ldk = ldk;
  eh.ks = const_cast<uint8_t*>(scale);
  eh.ldks = lds;
  // (by partials where that gains more than a launch: fp32, 14 rows, 1,088 x 1,152: 26.8 ->
  // 11.8 us; 39 rows, 1,426 x 1,490: 34.6 -> 16.4)
  const Shape whole = shape_of(type, gh.M, gh.N, gh.K, false, 4);
  const Shape split = shape_of(type, gh.M, gh.N, gh.K, true, 4);
  if (split.splits > 1 && split.us + 4.0 < whole.us) {
    gh.tile = split.tile;
    gh.splits = split.splits;
    gh.kh = INT_MAX;
    eh.part = c->at<float>(l.part);
    eh.ldp = gh.M;
    gated_dh_split(L, type, gh, eh);
  } else {
    ranged(gh, type, false, 4, [&](const GGemm& g) { gated_dh(L, type, g, eh); });
  }

  gx.B = eh.dgu;
  gx.ldb = eh.lddgu;
  gx.kh = Fp;
  gd.A = eh.h;
  gd.lda = c->ldh();
  gw.B = (const char*)eh.dgu + (dWg ? 0 : (size_t)Fp * es);
  gw.ldb = eh.lddgu;
  grads_shapes(type, dup, c->part_floats(c->Rws), &all);
  float* part = c->at<float>(l.part);
  for (int i = 0; i < 3; ++i) {
    GGemm& g = all.g[i];
    GEpi& e = all.e[i];
    const int join = i == 0 ? dup : 0;
    if (e.out && all.share) {
      all.part = e.part = part;
      e.ldp = tile_m(g.tile);
      f[n++] = {g, e, 0, all.share, all.work[i]};
    }
    if (!e.out || all.share || (g.splits == 1 && !join)) continue;
    e.part = part;
    e.ldp = g.M;
    part += (size_t)g.splits * up(g.N, VTILE) * g.M;
    f[n++] = {g, e, join, 0, 0};
  }
  gated_grads(L, type, all);
  gated_finish(L, type, type, f, n);
  return end(c);
}

int hf_gated_pack(hf_gated* c, const void* X, int64_t ldx, int64_t rows, int64_t cols,
                  int8_t* codes, int64_t ldc, uint8_t* scale, int64_t lds) {
  int rc;
  if (!c) return HF_EINVAL;
  if ((rc = check_size(c, rows, HF_GATED_MAX_ROWS, cols)) ||
      (rc = check_mat(c, X, ldx, cols, c->es, rows, "X")) ||
      (rc = check_mat(c, codes, ldc, cols, 1, rows, "codes")) ||
      (rc = check_mat(c, scale, lds, blocks_of(cols), 1, rows, "scale")) ||
      (rc = check_apart(c, X, "X", codes, "codes", rows)) || (rc = follow(c, true)))
    return rc;
  gated_pack(Launch{c->stream, nullptr}, c->type, X, ldx, rows, (int)cols, codes, ldc, scale, lds);
  return end(c);
}

int hf_gated_unpack(hf_gated* c, const int8_t* codes, int64_t ldc, const uint8_t* scale,
                    int64_t lds, int64_t rows, int64_t cols, void* X, int64_t ldx) {
  int rc;
  if (!c) return HF_EINVAL;
  if ((rc = check_size(c, rows, HF_GATED_MAX_ROWS, cols)) ||
      (rc = check_mat(c, codes, ldc, cols, 1, rows, "codes")) ||
      (rc = check_mat(c, scale, lds, blocks_of(cols), 1, rows, "scale")) ||
      (rc = check_mat(c, X, ldx, cols, c->es, rows, "X")) ||
      (rc = check_apart(c, codes, "codes", X, "X", rows)) || (rc = follow(c, true)))
    return rc;
  gated_unpack(Launch{c->stream, nullptr}, c->type, codes, ldc, scale, lds, rows, (int)cols, X, ldx);
  return end(c);
}

int hf_gated_codes(hf_gated* c, const void* X, int64_t ldx, int64_t rows, int64_t cols,
                   int8_t* codes, int64_t ldc, float* scale) {
  int rc;
  if (!c) return HF_EINVAL;
  if ((rc = check_size(c, rows, HF_GATED_MAX_OUT, cols)) ||
      (rc = check_mat(c, X, ldx, cols, c->es, rows, "X")) ||
      (rc = check_mat(c, codes, ldc, cols, 1, rows, "codes")) ||
      (rc = check_mat(c, scale, 1, 1, 4, rows, "scale")) ||
      (rc = check_apart(c, X, "X", codes, "codes", rows)) || (rc = follow(c, true)))
    return rc;
  gated_codes(Launch{c->stream, nullptr}, c->type, X, ldx, rows, (int)cols, codes, ldc, (int)cols,
              scale);
  return end(c);
}

int hf_gated_product(hf_gated* c, const int8_t* A, int64_t lda, const float* sa, const int8_t* B,
                     int64_t ldb, const float* sb, int64_t rows, int64_t n, int64_t k, void* Y,
                     int64_t ldy) {
  int rc;
  if (!c) return HF_EINVAL;
  if ((rc = check_rows(c, rows))) return rc;
  if (n < 1 || n > HF_GATED_MAX_OUT)
    return fail(c, HF_EINVAL, "%lld channels outside [1, %d]", (long long)n, HF_GATED_MAX_OUT);
  if (k < 1 || k > std::max(c->D, c->F))
    return fail(c, HF_EINVAL, "%lld columns outside [1, %d], the larger of the widths",
                (long long)k, std::max(c->D, c->F));
  if ((rc = check_mat(c, A, lda, k, 1, rows, "A")) || (rc = check_mat(c, sa, 1, 1, 4, rows, "sa")) ||
      (rc = check_mat(c, B, ldb, k, 1, n, "B")) || (rc = check_mat(c, sb, 1, 1, 4, n, "sb")) ||
      (rc = check_mat(c, Y, ldy, n, c->es, rows, "Y")) ||
      (rc = check_apart(c, A, "A", Y, "Y", rows)) || (rc = check_apart(c, B, "B", Y, "Y", rows)) ||
      (rc = check_ready(c, rows)) || (rc = follow(c, true)))
    return rc;
  if (rows == 0) return HF_OK;
  const Launch L{c->stream, nullptr};
  const Layout& l = c->lay;
  const int T = (int)rows, K = (int)up(k, CPAD);
  const bool place = k % CPAD == 0 && loads16(B, ldb, 1);
  if (T <= (place ? FEW_DOWN : FEW_X)) {
    GGemm g = product((int)n, T, (int)k);
    GEpi e = epilogue(c, T);
    operands(&g, B, ldb, nullptr, 0, A, lda);
    e.sn = sa;
    e.sm = sb;
    set_out(&e, Y, ldy, T, (int)n);
    if (T == 1 && k > ONE_BYTES) gated_one_down(L, VT_I8, c->type, g, e);
    else gated_few_down(L, VT_I8, c->type, g, e);
    return end(c);
  }
  // channels at a time: of those where they are as many as a launch takes with the most
  // rows (fewer than 2^32 work-items), or as many as are packed
  const int64_t step = place ? (int64_t)1 << 19
                             : std::max<int64_t>((int64_t)(WPACK_BYTES / (size_t)K) / 256 * 256, 256);
  long long ldaq = 0;
  const void* aq = nullptr;
  for (int64_t n0 = 0; n0 < n; n0 += step) {
    const int nn = (int)std::min(step, n - n0);
    Pads pads;
    GGemm g = product((int)up(nn, 64), T, K);
    if (n0 == 0)
      aq = pads.operand(k % CPAD == 0 && loads16(A, lda, 1), A, lda, T, (int)k, 1,
                        c->at<void>(l.aq), T, K, 1, &ldaq);
    g.A = pads.operand(place, B + n0 * ldb, ldb, nn, (int)k, 1, c->at<void>(l.bq), nn, K, 1, &g.lda);
    g.alim = nn;
    g.B = aq;
    g.ldb = ldaq;
    gated_pad(L, pads.all);
    GEpi e = epilogue(c, T);
    e.sn = sa;
    e.sm = sb + n0;
    set_out(&e, (char*)Y + n0 * c->es, ldy, T, nn);
    summed(c, L, VT_I8, c->type, g, e, 0, 4, [&](const GGemm& gg, const GEpi& ee) {
      gated_down(L, VT_I8, c->type, gg, ee);
    });
  }
  return end(c);
}

int hf_gated_forward_codes(hf_gated* c, const void* X, int64_t ldx, const int8_t* Wg, int64_t ldg,
                           const float* sg, const int8_t* Wu, int64_t ldu, const float* su,
                           const int8_t* Wd, int64_t ldd, const float* sd, int64_t rows, void* Y,
                           int64_t ldy) {
  int rc;
  if (!c) return HF_EINVAL;
  if ((rc = check_rows(c, rows)) ||
      (rc = check_mat(c, X, ldx, c->D, c->es, rows, "X")) ||
      (rc = check_weights(c, Wg, ldg, Wu, ldu, Wd, ldd, 1)) ||
      (rc = check_mat(c, sg, 1, 1, 4, c->F, "sg")) || (rc = check_mat(c, su, 1, 1, 4, c->F, "su")) ||
      (rc = check_mat(c, sd, 1, 1, 4, c->D, "sd")) ||
      (rc = check_mat(c, Y, ldy, c->D, c->es, rows, "Y")) ||
      (rc = check_apart(c, X, "X", Y, "Y", rows)) ||
      (rc = check_ready(c, rows)) || (rc = follow(c, true)))
    return rc;
  if (rows == 0) return HF_OK;
  const Launch L{c->stream, nullptr};
  const Layout& l = c->lay;
  const int T = (int)rows, D = c->D, F = c->F, Dc = c->Dc, Fc = c->Fc, Fp = c->Fp;
  int8_t* xq = c->at<int8_t>(l.xq);
  int8_t* hq = c->at<int8_t>(l.hq);
  float *sx = c->at<float>(l.sx), *sh = c->at<float>(l.sh);
  const bool few = T <= FEW_X, place = F == Fc && loads16(Wd, ldd, 1);
  const bool few_down = few && (T <= FEW_DOWN || !place);
  GGemm gu = few ? product(F, T, D) : product(2 * Fp, T, Dc);
  GGemm gd = few_down ? product(D, T, F) : product(c->Dp, T, Fc);
  GEpi eu = epilogue(c, T), ed = epilogue(c, T);
  gd.alim = D;
  if (few) {
    operands(&gu, Wg, ldg, Wu, ldu, xq, c->ldxq());
    operands(&gd, Wd, ldd, nullptr, 0, hq, c->ldhq());
  } else {
    Pads pads;
    const bool pair = D == Dc && ldg == ldu && loads16(Wg, ldg, 1) && loads16(Wu, ldu, 1);
    gu.A = pads.operand(pair, Wg, ldg, F, D, 1, c->at<void>(l.wg), F, Dc, 1, &gu.lda);
    gu.A1 = pads.operand(pair, Wu, ldu, F, D, 1, c->at<void>(l.wu), F, Dc, 1, &gu.lda);
    gu.alim = F;
    gu.B = xq;
    gu.ldb = c->ldxq();
    gd.A = pads.operand(place, Wd, ldd, D, F, 1, c->at<void>(l.wd), D, Fc, 1, &gd.lda);
    gd.B = hq;
    gd.ldb = c->ldhq();
    gated_pad(L, pads.all);
  }
  gated_codes(L, c->type, X, ldx, T, D, xq, c->ldxq(), Dc, sx);
  eu.sn = sx;
  eu.sm = sg;
  eu.sm1 = su;
  eu.h = c->at<float>(l.hf);
  eu.ldh = Fc;
  eu.hmax = c->at<float>(l.hmax);
  eu.ldmax = few ? (F + 15) / 16 : Fp / 32;
  const bool one_up = T == 1 && D > ONE_BYTES;
  if (one_up) {
    gated_one_up(L, VT_I8, gu, eu);
  } else if (few) {
    gated_few_up(L, VT_I8, gu, eu);
  } else {
    ranged(gu, VT_I8, false, 3, [&](const GGemm& g) { gated_up(L, VT_I8, g, eu); });
  }
  if (one_up) gated_codes_h(L, (float*)eu.h, Fc, (float*)eu.h, Fc, F, T, F, hq, c->ldhq(), Fc, sh);
  else gated_codes_h(L, (float*)eu.h, Fc, eu.hmax, eu.ldmax, eu.ldmax, T, F, hq, c->ldhq(), Fc, sh);
  ed.sn = sh;
  ed.sm = sd;
  set_out(&ed, Y, ldy, T, D);
  if (T == 1 && F > ONE_BYTES) {
    gated_one_down(L, VT_I8, c->type, gd, ed);
  } else if (few_down) {
    gated_few_down(L, VT_I8, c->type, gd, ed);
  } else {
    summed(c, L, VT_I8, c->type, gd, ed, 0, 4, [&](const GGemm& g, const GEpi& e) {
      gated_down(L, VT_I8, c->type, g, e);
    });
  }
  return end(c);
}

const char* hf_gated_last_error(const hf_gated* c) {
  return c ? c->err.c_str() : "null context";
}

}  // extern "C"
