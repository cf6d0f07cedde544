// Checks on the host what every launch of the gated block's calls reads and writes:
// the launchers are replaced by ones that work out the kernels' ranges from their
// arguments, each of which has to lie in one array of the call or in one part of the
// workspace.  Addresses are made up and never read through.
#include "gated_api.cpp"

#include <cstdio>
#include <cstdlib>
#include <map>
#include <random>
#include <string>
#include <vector>

namespace {
struct Area {
  size_t bytes;
  std::string name;
};
std::map<size_t, Area> areas;       // by first address
std::string call;
long checked = 0;

void within(const char* what, const void* p, size_t bytes, int align = 1) {
  ++checked;
  if (!bytes) return;
  const size_t at = (size_t)p;
  auto it = areas.upper_bound(at);
  const bool any = it != areas.begin();
  if (any) --it;
  if (!any || at + bytes > it->first + it->second.bytes || at % align) {
    printf("%s: %s: %zu bytes from %zu of %s, which has %zu\n", call.c_str(), what, bytes,
           any ? at - it->first : at, any ? it->second.name.c_str() : "nothing",
           any ? it->second.bytes : 0);
    exit(1);
  }
}
void equal(const char* what, long long a, long long b) {
  if (a == b) return;
  printf("%s: %s: %lld, not %lld\n", call.c_str(), what, a, b);
  exit(1);
}
// rows x cols elements of es bytes, ld apart
void rect(const char* what, const void* p, long long rows, long long ld, long long cols, int es,
          int align = 1) {
  if (rows < 1 || cols < 1) return;
  within(what, p, ((size_t)(rows - 1) * ld + cols) * es, align);
  if (rows > 1) within(what, (const char*)p + (size_t)ld * es, (size_t)cols * es, align);
}
size_t part_floats(const GGemm& g, const GEpi& e) {
  const long long rn = tile_n(g.tile), gy = (g.N + rn - 1) / rn;
  return ((size_t)(g.splits - 1) * gy * rn + g.N - 1) * e.ldp + (g.M - g.m0);
}
// output of "down" and the gradients: partials or out
void results(const GGemm& g, const GEpi& e, int es) {
  if (e.part) {
    within("partials", e.part, part_floats(g, e) * 4, 16);
    within("partials' rows", (const float*)e.part + e.ldp, 16, 16);
    return;
  }
  rect("out", e.out, e.nout, e.ldo, e.mout, es);
  if (e.n1 < g.N) rect("out1", e.out1, e.nout, e.ldo1, e.mout, es);
}
}  // namespace

namespace hfk {
void gated_up(const Launch&, int type, const GGemm& g, const GEpi& e) {
  const int es = es_of(type);
  rect("A", g.A, g.alim, g.lda, g.K, es, 16);
  rect("A1", g.A1, g.alim, g.lda, g.K, es, 16);
  rect("X", g.B, g.blim, g.ldb, g.K, es, 16);
  rect("h", e.h, e.T + e.dup, e.ldh, e.Fp, es == 2 ? 2 : 4, 16);
  if (es == 1) {
    rect("hmax", e.hmax, e.T, e.ldmax, e.Fp / 32, 4);
    within("scales", e.sm, e.F * 4);
    within("scales", e.sm1, e.F * 4);
    within("scales", e.sn, e.T * 4);
  }
  if (e.keep == KEEP_FULL) rect("kept", e.kept, e.T, e.ldk, 2 * e.F, es);
  if (e.keep == KEEP_CODES) {
    rect("kept", e.kept, e.T, e.ldk, 2 * e.F, 1);
    rect("kept's scale", e.ks, e.T, e.ldks, 2 * blocks_of(e.F), 1);
  }
}
void gated_down(const Launch&, int type, int out_type, const GGemm& g, const GEpi& e) {
  const int es = es_of(type);
  rect("Wd", g.A, g.alim, g.lda, g.K, es, 16);
  rect("h", g.B, g.blim, g.ldb, g.K, es, 16);
  if (es == 1 && !e.part) {
    within("scales", e.sm, e.mout * 4);
    within("scales", e.sn, e.nout * 4);
  }
  results(g, e, es_of(out_type));
}
static void few(int type, int out_type, const GGemm& g, const GEpi& e, bool up, bool one) {
  const int es = es_of(type), h32 = up && (es != 2 || e.h32);
  rect("A", g.A, g.M, g.lda, g.K, es);
  if (up) rect("A1", g.A1, g.M, g.lda1, g.K, es);
  // (h of one row is fp32)
  const bool two = !up && !one && es == 2 && g.N <= TWO_X;
  rect("B", g.B, g.N + (two ? e.dup : 0), g.ldb, g.K, !up && one && es == 2 ? 4 : es);
  if (es == 1) {
    within("scales", e.sm, g.M * 4);
    within("scales", e.sn, g.N * 4);
    if (up) within("scales", e.sm1, g.M * 4);
  }
  if (!up) return rect("out", e.out, e.nout, e.ldo, e.mout, es_of(out_type));
  rect("h", e.h, e.T + (h32 ? 0 : e.dup), e.ldh, one ? e.F : e.Fp, h32 ? 4 : es, 8);
  if (es == 1 && !one) rect("hmax", e.hmax, e.T, e.ldmax, (e.F + 15) / 16, 4);
  if (e.keep == KEEP_FULL) rect("kept", e.kept, e.T, e.ldk, 2 * e.F, es);
  if (e.keep == KEEP_CODES) rect("g and u", e.kept, e.T, e.ldk, 2 * e.F, 4);
}
void gated_few_up(const Launch&, int type, const GGemm& g, const GEpi& e) {
  few(type, type, g, e, true, false);
}
void gated_few_down(const Launch&, int type, int out, const GGemm& g, const GEpi& e) {
  few(type, out, g, e, false, false);
}
void gated_one_up(const Launch&, int type, const GGemm& g, const GEpi& e) {
  few(type, type, g, e, true, true);
}
void gated_one_down(const Launch&, int type, int out, const GGemm& g, const GEpi& e) {
  few(type, out, g, e, false, true);
}
void gated_dh(const Launch&, int type, const GGemm& g, const GEpi& e) {
  const int es = es_of(type);
  rect("Wd", g.A, g.K, g.lda, g.M, es, 16);
  rect("dY", g.B, g.blim, g.ldb, g.K, es, 16);
  rect("h", e.h, g.N + e.dup, e.ldh, e.Fp, es, 16);
  rect("dg, du", e.dgu, g.N + e.dup, e.lddgu, 2 * e.Fp, es, 16);
  rect("kept", e.kept, e.T, e.ldk, 2 * e.F, e.keep == KEEP_FULL ? es : 1);
  if (e.keep == KEEP_CODES) rect("kept's scale", e.ks, e.T, e.ldks, 2 * blocks_of(e.F), 1);
}
void gated_dh_split(const Launch& L, int type, const GGemm& g, const GEpi& e) {
  gated_dh(L, type, g, e);
  within("partials", e.part, part_floats(g, e) * 4, 16);
  equal("one matrix", g.kh >= g.K, 1);
}
void gated_grads(const Launch&, int type, GGrads a) {
  const int es = es_of(type);
  const size_t tile = tile_m(a.g[0].tile) * tile_n(a.g[0].tile);
  if (a.share) {
    within("shares' partials", a.part, 2 * units_of(a.g[0].tile) * tile * 4, 16);
    int work = 0;
    for (int i = 0; i < 3; ++i) {
      equal("work", a.work[i], work);
      if (a.e[i].out) work += gated_tiles(a.g[i]) * (a.g[i].K * es / 128);
    }
    equal("work", a.work[3], work);
    equal("units", (work + a.share - 1) / a.share <= units_of(a.g[0].tile), 1);
  }
  for (int i = 0; i < 3; ++i) {
    const GGemm& g = a.g[i];
    GEpi e = a.e[i];
    if (a.share) e.part = nullptr;       // (whole tiles)
    if (!e.out) continue;
    if (i == 0) {
      rect("Wg", g.A, g.kh, g.lda, g.M, es, 16);
      rect("Wu", g.A1, g.K - g.kh, g.lda, g.M, es, 16);
      rect("dg, du", g.B, g.blim, g.ldb, g.K, es, 16);
    } else {
      rect("A", g.A, g.at ? std::min(g.K, g.ktail) : g.K, g.lda, g.M, es, 16);
      rect("B", g.B, g.bt ? std::min(g.K, g.ktail) : g.K, g.ldb, g.N, es, 16);
      if (g.at) rect("A's tail", g.at, g.K - g.ktail, g.ldat, g.M, es, 16);
      if (g.bt) rect("B's tail", g.bt, g.K - g.ktail, g.ldbt, g.N, es, 16);
    }
    results(g, e, es);
  }
}
void gated_finish(const Launch&, int type, int out_type, const GFinish* f, int n) {
  for (int i = 0; i < n; ++i) {
    const GGemm& g = f[i].g;
    GEpi e = f[i].e;
    if (f[i].share)
      within("shares' partials", e.part, 2 * units_of(g.tile) * (size_t)e.ldp * tile_n(g.tile) * 4, 16);
    else if (g.splits) within("partials", e.part, part_floats(g, e) * 4, 16);
    if (type == VT_I8) {
      within("scales", e.sm, e.mout * 4);
      within("scales", e.sn, e.nout * 4);
    }
    e.part = nullptr;
    results(g, e, es_of(out_type));
  }
}
void gated_pad(const Launch&, const GPads& p) {
  if (p.n > GPADS) within("copies", nullptr, 1);
  for (int i = 0; i < p.n; ++i) {
    const GPad& q = p.p[i];
    rect("source", q.src, q.rows, q.ld, q.cols, q.scale ? 1 : q.es);
    if (q.scale) rect("source's scale", q.scale, q.rows, q.lds, blocks_of(q.cols), 1);
    rect("copy", q.dst, (long long)q.prows * q.times, q.pcols, q.pcols, q.es, 16);
  }
}
void gated_pack(const Launch&, int type, const void* X, long long ldx, long long rows, int cols,
                int8_t* codes, long long ldc, uint8_t* scale, long long lds) {
  rect("X", X, rows, ldx, cols, es_of(type));
  rect("codes", codes, rows, ldc, cols, 1);
  rect("scale", scale, rows, lds, blocks_of(cols), 1);
}
void gated_unpack(const Launch& L, int type, const int8_t* codes, long long ldc,
                  const uint8_t* scale, long long lds, long long rows, int cols, void* X,
                  long long ldx) {
  gated_pack(L, type, X, ldx, rows, cols, const_cast<int8_t*>(codes), ldc,
             const_cast<uint8_t*>(scale), lds);
}
void gated_codes(const Launch&, int type, const void* X, long long ldx, long long rows, int cols,
                 int8_t* codes, long long ldc, int zcols, float* scale) {
  rect("X", X, rows, ldx, cols, es_of(type));
  rect("codes", codes, rows, ldc, zcols, 1);
  within("scale", scale, rows * 4);
}
void gated_codes_h(const Launch&, const float* H, long long ldh, const float* hmax,
                   long long ldmax, int nmax, int rows, int cols, int8_t* codes, long long ldc,
                   int zcols, float* scale) {
  rect("h", H, rows, ldh, cols, 4);
  rect("hmax", hmax, rows, ldmax, nmax, 4);
  rect("codes", codes, rows, ldc, zcols, 1);
  within("scale", scale, rows * 4);
}
}  // namespace hfk

namespace {
constexpr size_t APART = (size_t)1 << 44;
size_t next = 0;
std::mt19937 rng(1);
int64_t below(int64_t n) { return (int64_t)(rng() % (uint64_t)n); }
struct Mat {
  void* p;
  int64_t ld;
};
// a rows x cols array, contiguous, or rows apart and `shift` elements in
Mat mat(const char* name, int64_t rows, int64_t cols, int es, bool odd) {
  const int64_t ld = cols + (odd ? 1 + below(9) : 0), shift = odd ? 1 + below(3) : 0;
  next += APART;
  areas[next] = {(size_t)(rows * ld + shift) * es, name};
  return {(void*)(next + shift * es), ld};
}
// the parts of a workspace that a kind of call uses
void parts(const hf_gated* c, std::initializer_list<size_t> offsets) {
  std::vector<size_t> at(offsets);
  at.push_back(c->lay.need);
  for (size_t i = 0; i + 1 < at.size(); ++i)
    if (at[i + 1] > at[i]) areas[(size_t)c->ws + at[i]] = {at[i + 1] - at[i], "workspace part " + std::to_string(i)};
}
void ok(int rc, const hf_gated* c) {
  if (rc == HF_OK) return;
  printf("%s: %d %s\n", call.c_str(), rc, hf_gated_last_error(c));
  exit(1);
}
void run(int64_t T, int D, int F, int type, bool odd, int64_t n) {
  hf_gated* c = nullptr;
  if (hf_gated_create(D, F, HF_SILU, type, T, nullptr, &c) != HF_OK) exit(1);
  const int es = es_of(type);
  char* ws = (char*)APART;
  ok(hf_gated_set_workspace(c, ws, hf_gated_workspace_bytes(c, T)), c);
  const Layout& l = c->lay;
  auto named = [&](const char* what) {
    char b[200];
    snprintf(b, sizeof b, "%s: %lld rows, %d x %d, type %d%s, %lld channels", what, (long long)T, D,
             F, type, odd ? ", rows apart" : "", (long long)n);
    call = b;
    areas.clear();
    next = APART;
  };
  const int64_t nb = (F + 31) / 32;
  for (int keep = 0; keep < 3; ++keep) {
    named("forward");
    parts(c, {l.part, l.wg, l.wu, l.wd, l.xp, l.yp, l.xt, l.yt, l.h, l.dgu, l.gu});
    Mat X = mat("X", T, D, es, odd), Wg = mat("Wg", F, D, es, odd), Wu = mat("Wu", F, D, es, odd),
        Wd = mat("Wd", D, F, es, odd), Y = mat("Y", T, D, es, odd),
        k = mat("kept", T, 2 * F, keep == 2 ? 1 : es, odd), s = mat("scale", T, 2 * nb, 1, odd);
    ok(hf_gated_forward(c, X.p, X.ld, Wg.p, Wg.ld, Wu.p, Wu.ld, Wd.p, Wd.ld, T, Y.p, Y.ld, keep,
                        k.p, k.ld, (uint8_t*)s.p, s.ld), c);
    if (!keep) continue;
    Mat dY = mat("dY", T, D, es, odd), dX = mat("dX", T, D, es, odd), dG = mat("dWg", F, D, es, odd),
        dU = mat("dWu", F, D, es, odd), dD = mat("dWd", D, F, es, odd);
    Mat xc = mat("X's codes", T, D, 1, odd), xs = mat("X's scale", T, (D + 31) / 32, 1, odd);
    for (int need = 1; need < 16; need += keep == 1 ? 1 : 14) {
      named("gradient");       // (same arrays)
      parts(c, {l.part, l.wg, l.wu, l.wd, l.xp, l.yp, l.xt, l.yt, l.h, l.dgu, l.gu});
      X = mat("X", T, D, es, odd), Wg = mat("Wg", F, D, es, odd), Wu = mat("Wu", F, D, es, odd),
      Wd = mat("Wd", D, F, es, odd), k = mat("kept", T, 2 * F, keep == 2 ? 1 : es, odd),
      s = mat("scale", T, 2 * nb, 1, odd), dY = mat("dY", T, D, es, odd),
      dX = mat("dX", T, D, es, odd), dG = mat("dWg", F, D, es, odd), dU = mat("dWu", F, D, es, odd),
      dD = mat("dWd", D, F, es, odd), xc = mat("X's codes", T, D, 1, odd),
      xs = mat("X's scale", T, (D + 31) / 32, 1, odd);
      const bool coded = keep == 2;
      ok(hf_gated_grad(c, coded ? xc.p : X.p, coded ? xc.ld : X.ld, coded ? (uint8_t*)xs.p : nullptr,
                       xs.ld, Wg.p, Wg.ld, Wu.p, Wu.ld, Wd.p, Wd.ld, keep, k.p, k.ld,
                       (uint8_t*)s.p, s.ld, dY.p, dY.ld, T, need & 1 ? dX.p : nullptr, dX.ld,
                       need & 2 ? dG.p : nullptr, dG.ld, need & 4 ? dU.p : nullptr, dU.ld,
                       need & 8 ? dD.p : nullptr, dD.ld, 0), c);
    }
  }
  {
    named("forward of codes");
    parts(c, {l.part, l.wg, l.wu, l.wd, l.xq, l.sx, l.hf, l.hmax, l.hq, l.sh});
    Mat X = mat("X", T, D, es, odd), Wg = mat("Wg", F, D, 1, odd), Wu = mat("Wu", F, D, 1, odd),
        Wd = mat("Wd", D, F, 1, odd), Y = mat("Y", T, D, es, odd), sg = mat("sg", F, 1, 4, false),
        su = mat("su", F, 1, 4, false), sd = mat("sd", D, 1, 4, false);
    ok(hf_gated_forward_codes(c, X.p, X.ld, (int8_t*)Wg.p, Wg.ld, (float*)sg.p, (int8_t*)Wu.p, Wu.ld,
                              (float*)su.p, (int8_t*)Wd.p, Wd.ld, (float*)sd.p, T, Y.p, Y.ld), c);
  }
  for (int64_t k : {(int64_t)std::max(D, F), (int64_t)1 + below(std::max(D, F))}) {
    named("product");
    parts(c, {l.part, l.wg, l.wu, l.wd, l.aq, l.bq});
    Mat A = mat("A", T, k, 1, odd), B = mat("B", n, k, 1, odd), Y = mat("Y", T, n, es, odd),
        sa = mat("sa", T, 1, 4, false), sb = mat("sb", n, 1, 4, false);
    ok(hf_gated_product(c, (int8_t*)A.p, A.ld, (float*)sa.p, (int8_t*)B.p, B.ld, (float*)sb.p, T, n, k,
                        Y.p, Y.ld), c);
  }
  hf_gated_destroy(c);
}
}  // namespace

// cases: how many at random
int main(int, char** argv) {
  for (int64_t T : {1, 16, 17, 64, 65, 128, 129, 1000, 8192})
    for (int D : {1, 64, 1000, 4096})
      for (int F : {1, 64, 1365, 16384})
        for (int type : {0, 1}) run(T, D, F, type, (D + F + T) % 3 == 0, 1 + 37 * D);
  const int cases = atoi(argv[1]);
  for (int i = 0; i < cases; ++i) {
    // sizes over all scales, half of them whole blocks
    auto size = [&](int bits) {
      const int64_t top = (int64_t)1 << below(bits + 1), v = top + below(top);
      return std::min(below(2) ? up(v, 128) : v, (int64_t)1 << bits);
    };
    const int64_t T = size(18), D = size(16), F = size(16);
    run(T, (int)D, (int)F, (int)below(2), below(3) == 0, size(22));
  }
  printf("%ld ranges\n", checked);
  return 0;
}
