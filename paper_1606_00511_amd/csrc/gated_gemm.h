// The products of the gated feed-forward block (T rows, width D, hidden F):
//   up    g = X Wg^T, u = X Wu^T and h = phi(g) u, which leaves the tile; g and
//         u only where they are kept for the gradient
//   down  Y = h Wd^T
//   dh    dh = dY Wd, which stays in the tile: h, dg = dh u phi'(g) and
//         du = dh phi(g) leave it
//   dx    dX = dg Wg + du Wu, one product of 2 F
//   dw    dWd = dY^T h, and dWg = dg^T X with dWu = du^T X as one product
// 2 T D F operations for each of the three matrices forward and four times that
// backward: bound by the matrix cores, and for few rows by reading the matrices.
//
// A tile of "up" takes its rows m from both matrices, 32 of Wg and the same 32 of
// Wu in turn: a wave then has g and u of the same features in neighbouring blocks
// of its accumulators, and neither goes through memory.
// Sums are fp32 (codes: int32, exact), the activation and its slope fp32; h, dg
// and du are rounded to the type for the products that read them (few bf16
// rows: to two terms of it, which cost little where the matrices bound a product).
#pragma once

#include "gated_act.h"
#include "gated_values.h"
#include "mfma_tile.h"

namespace hfk {
namespace {

enum { UP, DOWN, DH, DX, DW };

// h, dg or du to the workspace, where whole chunks are aligned; dup: the rest of
// the rounding too
__device__ __forceinline__ void put_term(float* p, const float (&v)[8], long long) {
  *(f32x4*)p = f32x4{v[0], v[1], v[2], v[3]};
  *(f32x4*)(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
}
__device__ __forceinline__ void put_term(bf16_t* p, const float (&v)[8], long long rest) {
  const u32x4 w = f2bf8(v);
  *(u32x4*)p = w;
  if (!rest) return;
  float left[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) left[j] = rest_of(v[j], j & 1 ? w[j / 2] >> 16 : w[j / 2] & 0xffffu);
  *(u32x4*)(p + rest) = f2bf8(left);
}

// what a wave has written to its own part of LDS is there for its other lanes
__device__ __forceinline__ void staged_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}
// 8 numbers of row r of a wave's staged part, from its chunk c of 4 on
template <int RL>
__device__ __forceinline__ void staged8(const float* s, int r, int c, float (&v)[8]) {
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const f32x4 w = *(const f32x4*)(s + r * RL + 4 * ((c + k) ^ (r & (RL / 4 - 1))));
#pragma unroll
    for (int j = 0; j < 4; ++j) v[4 * k + j] = w[j];
  }
}

// rows n0 .. n0 + 31 of "up": WM / 2 blocks of 32 features from f0, g and u in
// turn in the staged columns.  FULL: all of these rows and features exist.
template <class E, int WM, int ACT, bool FULL>
__device__ __forceinline__ void up_rows(const float* s, int lane, const GEpi& e, int n0, int f0,
                                        const float (&sg)[8], const float (&su)[8]) {
  constexpr int RL = 32 * WM, FC = 2 * WM;       // lanes a row, 8 features each
  constexpr bool I8 = sizeof(E) == 1;
  const int fc = lane % FC, f = f0 + 8 * fc, c = 16 * (fc / 4) + 2 * (fc % 4);
  const int have = FULL ? 8 : e.F - f;           // < 8: the last of them
  if (!FULL && f >= e.Fp) return;                // (the same in the lanes of a block)
#pragma unroll FULL ? 2 : 1
  for (int i = 0; i < FC / 2; ++i) {
    const int r = (lane + 64 * i) / FC, n = n0 + r;
    if (!FULL && n >= e.T) break;
    float g[8], u[8], hv[8];
    staged8<RL>(s, r, c, g);
    staged8<RL>(s, r, c + 8, u);
    if constexpr (I8) {
      const RowFactor sn(e.sn[n]);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        g[j] = sn.scaled(__float_as_int(g[j]), sg[j]);
        u[j] = sn.scaled(__float_as_int(u[j]), su[j]);
      }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      hv[j] = act_of<ACT, sizeof(E) != 2>(g[j]) * u[j];
      if (!FULL && j >= have) hv[j] = 0.0f;
    }
    if constexpr (I8) {
      put_term((float*)e.h + (size_t)n * e.ldh + f, hv, 0);
      uint32_t big = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) big = max(big, __float_as_uint(hv[j]) & 0x7fffffffu);
      big = max(big, (uint32_t)__shfl_xor((int)big, 1, 64));
      big = max(big, (uint32_t)__shfl_xor((int)big, 2, 64));
      if (fc % 4 == 0) e.hmax[(size_t)n * e.ldmax + f / 32] = __uint_as_float(big);
    } else {
      put_term((E*)e.h + (size_t)n * e.ldh + f, hv, e.dup * e.ldh);
      if (e.keep == KEEP_FULL) {
        E* p = (E*)e.kept + (size_t)n * e.ldk + f;
        put(p, g, have);
        put(p + e.F, u, have);
      } else if (e.keep == KEEP_CODES) {
        int8_t* p = (int8_t*)e.kept + (size_t)n * e.ldk + f;
        uint8_t* ks = e.ks + (size_t)n * e.ldks + f / CODE_BLOCK;
        const int bg = put_codes(p, g, have), bu = put_codes(p + e.F, u, have);
        if (fc % 4 == 0 && have > 0) {
          ks[0] = (uint8_t)bg;
          ks[(e.F + CODE_BLOCK - 1) / CODE_BLOCK] = (uint8_t)bu;
        }
      }
    }
  }
}

// What is kept of g and u at a lane's places in PB of its rows of 32 WM features, all
// of which exist: fetched ahead of the products that need it.
template <class E, bool CODES, int WM>
struct Kept {
  static constexpr int FC = 4 * WM, I = 2 * WM;  // lanes a row, 8 features each; rows a lane
  // rows at once, in 16 to 20 registers (twice as many leave the largest tiles none)
  static constexpr int PB = CODES ? (I < 4 ? I : 4) : sizeof(E) == 2 ? 2 : 1;
  static constexpr int W = CODES ? 2 : 2 * (int)sizeof(E);
  uint32_t g[PB][W], u[PB][W];
  uint8_t sg[PB], su[PB];
  // rows n0 + (lane + 64 i) / FC, i = i0 .. i0 + PB - 1
  __device__ __forceinline__ void fetch(const GEpi& e, int lane, int n0, int i0, int f0) {
    const int f = f0 + 8 * (lane % FC), nb = (e.F + CODE_BLOCK - 1) / CODE_BLOCK;
#pragma unroll
    for (int i = 0; i < PB; ++i) {
      const int n = n0 + (lane + 64 * (i0 + i)) / FC;
      if constexpr (CODES) {
        const int8_t* p = (const int8_t*)e.kept + (size_t)n * e.ldk + f;
        const uint8_t* ks = e.ks + (size_t)n * e.ldks + f / CODE_BLOCK;
        __builtin_memcpy(g[i], p, 8);
        __builtin_memcpy(u[i], p + e.F, 8);
        sg[i] = ks[0];
        su[i] = ks[nb];
      } else {
        const E* p = (const E*)e.kept + (size_t)n * e.ldk + f;
#pragma unroll
        for (int j = 0; j < W; j += 4) {
          __builtin_memcpy(&g[i][j], (const char*)p + 4 * j, 16);
          __builtin_memcpy(&u[i][j], (const char*)(p + e.F) + 4 * j, 16);
        }
      }
    }
  }
  __device__ __forceinline__ void value(const uint32_t (&w)[W], uint8_t scale, float (&v)[8]) const {
    if constexpr (CODES) {
      const float step = code_step(scale);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = (float)(int8_t)(w[j >> 2] >> (8 * (j & 3))) * step;
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        v[j] = sizeof(E) == 4 ? __uint_as_float(w[j % W])
                              : bf2f(j & 1 ? w[j / 2] >> 16 : w[j / 2] & 0xffffu);
    }
  }
};

// h, dg and du of 8 features of a row from dh, g and u
template <class E, int ACT, bool FULL>
__device__ __forceinline__ void dh_chunk(const GEpi& e, int n, int f, int have, const float (&d)[8],
                                         float (&g)[8], float (&u)[8]) {
  float hv[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    float a, sl;
    act_and_slope<ACT, sizeof(E) == 4>(g[j], a, sl);
    hv[j] = a * u[j];
    g[j] = d[j] * u[j] * sl;
    u[j] = d[j] * a;
    if (!FULL && j >= have) hv[j] = g[j] = u[j] = 0.0f;
  }
  put_term((E*)e.h + (size_t)n * e.ldh + f, hv, e.dup * e.ldh);
  E* q = (E*)e.dgu + (size_t)n * e.lddgu + f;
  put_term(q, g, e.dup * e.lddgu);
  put_term(q + e.Fp, u, e.dup * e.lddgu);
}
// "dh" of a wave's 32 WN rows from n0 and 32 WM features from f0, all of which exist:
// stage(b) puts 32 rows of dh into s; what is kept of the next rows is on its way
// during the products of these
template <class E, bool CODES, int WM, int WN, int ACT, class Stage>
__device__ __forceinline__ void dh_full(const float* s, int lane, const GEpi& e, int n0, int f0,
                                        Stage stage) {
  typedef Kept<E, CODES, WM> K;
  constexpr int RL = 32 * WM, NB = K::I / K::PB;
  const int fc = lane % K::FC, f = f0 + 8 * fc;
  K first, other;
  first.fetch(e, lane, n0, 0, f0);
  __syncthreads();     // every wave is done with the operand stages
#pragma unroll
  for (int b = 0; b < WN; ++b) {
    stage(b);
#pragma unroll
    for (int q = 0; q < NB; ++q) {
      const int t = b * NB + q;
      K &k = t & 1 ? other : first, &next = t & 1 ? first : other;
      if (t + 1 < WN * NB) next.fetch(e, lane, n0 + 32 * ((t + 1) / NB), (t + 1) % NB * K::PB, f0);
#pragma unroll
      for (int i = 0; i < K::PB; ++i) {
        const int r = (lane + 64 * (q * K::PB + i)) / K::FC;
        float d[8], g[8], u[8];
        staged8<RL>(s, r, 2 * fc, d);
        k.value(k.g[i], k.sg[i], g);
        k.value(k.u[i], k.su[i], u);
        dh_chunk<E, ACT, true>(e, n0 + 32 * b + r, f, 8, d, g, u);
        __builtin_amdgcn_sched_barrier(0);     // (more of them at once take registers)
      }
    }
    staged_fence();
  }
}
// what is kept of row n's features from f on, of which there are `have`
template <class E>
__device__ __forceinline__ void get_kept(const GEpi& e, int n, int f, int have, float (&g)[8],
                                         float (&u)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) g[j] = u[j] = 0.0f;
  if (have <= 0) return;
  if (e.keep == KEEP_FULL) {
    const E* p = (const E*)e.kept + (size_t)n * e.ldk + f;
    get(p, g, have);
    get(p + e.F, u, have);
  } else {
    const int8_t* p = (const int8_t*)e.kept + (size_t)n * e.ldk + f;
    const uint8_t* ks = e.ks + (size_t)n * e.ldks + f / CODE_BLOCK;
    get_codes(p, code_step(ks[0]), g, have);
    get_codes(p + e.F, code_step(ks[(e.F + CODE_BLOCK - 1) / CODE_BLOCK]), u, have);
  }
}
// 32 rows from n0 of "dh", any below Np and of any features
template <class E, int WM, int ACT>
__device__ __forceinline__ void dh_rows(const float* s, int lane, const GEpi& e, int n0, int f0,
                                        int Np) {
  constexpr int RL = 32 * WM, FC = 4 * WM;
  const int fc = lane % FC, f = f0 + 8 * fc;
  if (f >= e.Fp) return;
#pragma unroll 1
  for (int i = 0; i < FC / 2; ++i) {
    const int r = (lane + 64 * i) / FC, n = n0 + r;
    if (n >= Np) break;
    const int have = n < e.T ? e.F - f : 0;
    float d[8], g[8], u[8];
    staged8<RL>(s, r, 2 * fc, d);
    get_kept<E>(e, n, f, have, g, u);
    dh_chunk<E, ACT, false>(e, n, f, have, d, g, u);
  }
}

// rows n0 .. n0 + 31 of a product of codes, scaled; sm: the columns' scales
template <class O, int RL>
__device__ __forceinline__ void scaled_part(const float* s, int lane, const GEpi& e, int n0, int m0,
                                            const float (&sm)[8]) {
  constexpr int CPR = RL / 8;
  const int c = lane % CPR, m = m0 + 8 * c, have = e.mout - m;
  if (have <= 0) return;
#pragma unroll
  for (int i = 0; i < CPR / 2; ++i) {
    const int r = (lane + 64 * i) / CPR, n = n0 + r;
    if (n >= e.nout) break;
    float v[8];
    staged8<RL>(s, r, 2 * c, v);
    const RowFactor sn(e.sn[n]);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = sn.scaled(__float_as_int(v[j]), sm[j]);
    put((O*)e.out + (size_t)n * e.ldo + m, v, have);
  }
}

// The stages of a workgroup, the same ones for every product that a kernel may compute.
template <class E, int N>
__device__ __forceinline__ E* stages() {
  __shared__ __attribute__((aligned(16))) E lds[N];
  return lds;
}

// A tile's share of K for a workgroup that has several in turn: nblk K blocks from vb0 on
// of tile (tm, tn), and where their partial goes, rows of the tile's columns; null: to the
// product's output.
struct Piece {
  int tid, tm, tn, vb0, nblk;
  float* part;
};
// The tile of workgroup L of product s, or (PIECE) what p says.  (Both are this function:
// with the other's tile handed over as a piece too, "up" of 8,192 rows, 4,096 x 16,384,
// took 1,865 us for 1,818.)
// E: the operands' type, O: the output's, ACT: the activation of "up" and "dh"
template <class E, class O, int MODE, int ACT, int WM, int WN, int GM, int GN, int S,
          bool PIECE = false>
__device__ __forceinline__ void ggemm_body(const GGemm& s, const GEpi& e, int L,
                                           const Piece& p = Piece()) {
  constexpr bool AKC = MODE == UP || MODE == DOWN, BKC = MODE != DW;
  constexpr int BK = 128 / (int)sizeof(E);
  constexpr int NW = GM * GN;
  constexpr int RM = 32 * WM * GM, RN = 32 * WN * GN;
  using TA = Tile<E, AKC, RM, BK, NW>;
  using TB = Tile<E, BKC, RN, BK, NW>;
  constexpr int EPC = TA::EPC;
  constexpr int STAGE = TA::SIZE + TB::SIZE;
  constexpr int ALL = S * STAGE;

  const int tid = PIECE ? p.tid : threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / GN, wn = wave % GN;
  const int li = lane & 31, h = lane >> 5;
  const int gx = (s.M - s.m0 + RM - 1) / RM, gy = (s.N + RN - 1) / RN;
  int tm = p.tm, tn = p.tn, tz = 0;
  if (!PIECE && !tile_at(L, gx, gy, s.splits, tm, tn, tz)) return;
  const int m0 = s.m0 + tm * RM, n0 = tn * RN;

  const int nvb = s.K / BK;
  int vb0 = 0, nblk = nvb;
  if (PIECE) {
    vb0 = p.vb0;
    nblk = p.nblk;
  } else if (s.splits > 1) {
    const int per = (nvb + s.splits - 1) / s.splits;
    vb0 = min(tz * per, nvb);
    nblk = min(nvb, vb0 + per) - vb0;
  }

  typename SumT<E>::T acc[WM][WN];
#pragma unroll
  for (int a = 0; a < WM; ++a)
#pragma unroll
    for (int b = 0; b < WN; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[a][b][r] = 0;

  // Element offsets of the lane's direct loads from the tile's origin.  Rows of
  // a K-contiguous operand past its last one read that one; chunks of a [k][m]
  // operand past its width read its last chunk (both feed outputs that are not
  // stored).
  const int fa = MODE == UP ? m0 / 2 : m0;       // A's first row or column
  const int ra = min(fa, s.alim - 1), rb = min(n0, s.blim - 1);   // (whole tiles may lie past it)
  auto offset_a = [&](int j, long long ld) {
    int row, ch;
    TA::src(wave, lane, j, row, ch);
    if (MODE == UP) row = row / 64 * 32 + row % 32;
    return AKC ? (uint32_t)((min(fa + row, s.alim - 1) - ra) * ld) + EPC * ch
               : (uint32_t)(row * ld) + min(EPC * ch, (s.M - 1 - m0) / EPC * EPC);
  };
  auto offset_b = [&](int j, long long ld) {
    int row, ch;
    TB::src(wave, lane, j, row, ch);
    return BKC ? (uint32_t)((min(n0 + row, s.blim - 1) - rb) * ld) + EPC * ch
               : (uint32_t)(row * ld) + min(EPC * ch, (s.N - 1 - n0) / EPC * EPC);
  };
  uint32_t offa[TA::INSTR], offb[TB::INSTR];
#pragma unroll
  for (int j = 0; j < TA::INSTR; ++j) offa[j] = offset_a(j, s.lda);
#pragma unroll
  for (int j = 0; j < TB::INSTR; ++j) offb[j] = offset_b(j, s.ldb);
  const size_t a0 = AKC ? (size_t)ra * s.lda : (size_t)m0;
  const size_t b0 = BKC ? (size_t)rb * s.ldb : (size_t)n0;
  const uint32_t lds0 = lds_address(stages<E, ALL>());
  static_assert(TA::CH == 8 || !AKC, "8 rows of 128 bytes a direct load");
  // direct load j of K block vb into stage st (A's, then B's)
  auto issue1 = [&](int vb, int st, int j) {
    const int k0 = vb * BK;
    const uint32_t base = lds0 + (uint32_t)sizeof(E) * (uint32_t)(st * STAGE);
    if (j < TA::INSTR) {
      const E* a = (const E*)s.A;
      int k = k0;
      // a load's 8 rows are of one matrix: blocks of 32 rows in turn
      if (MODE == UP && ((wave * TA::INSTR + j) / 4 & 1)) a = (const E*)s.A1;
      if (MODE == DX && k0 >= s.kh) {
        a = (const E*)s.A1;
        k -= s.kh;
      }
      a += a0 + (AKC ? (size_t)k : (size_t)k * s.lda) + offa[j];
      if (MODE == DW && s.at && k0 >= s.ktail)
        a = (const E*)s.at + a0 + (size_t)(k0 - s.ktail) * s.ldat + offset_a(j, s.ldat);
      dma16_at(a, base + (uint32_t)sizeof(E) * TA::dst(wave, j));
    } else {
      j -= TA::INSTR;
      const E* b = (const E*)s.B + b0 + (BKC ? (size_t)k0 : (size_t)k0 * s.ldb) + offb[j];
      if (MODE == DW && s.bt && k0 >= s.ktail)
        b = (const E*)s.bt + b0 + (size_t)(k0 - s.ktail) * s.ldbt + offset_b(j, s.ldbt);
      dma16_at(b, base + (uint32_t)sizeof(E) * (TA::SIZE + TB::dst(wave, j)));
    }
  };
  auto fetch1 = [&](FragsT<E, TA, TB, WM, WN>& f, int st, int q, int i) {
    const E* la = stages<E, ALL>() + st * STAGE;
    const E* lb = la + TA::SIZE;
    if (i < WN) f.b[i] = TB::frag(lb, wn * 32 * WN + 32 * i, lane, q);
    else f.a[i - WN] = TA::frag(la, wm * 32 * WM + 32 * (i - WN), lane, q);
  };
  k_loop<E, TA, TB, WM, WN, S>(acc, vb0, nblk, fetch1, issue1, [] {}, [](int) {});

  // Lane (li, h), register r of block (a, b) holds n = 32 b + li and
  // m = 32 a + 8 (r / 4) + 4 h + r % 4 of the wave's part of the tile.
  const int mt = m0 + wm * 32 * WM, nt = n0 + wn * 32 * WN;
  constexpr int RL = 32 * WM;
  static_assert(NW * 32 * RL * 4 <= S * STAGE * (int)sizeof(E), "staging exceeds the stages");
  float* const mine = (float*)stages<E, ALL>() + wave * 32 * RL;
  const bool parts = (MODE == DOWN || MODE == DX || MODE == DW) && (PIECE ? p.part : e.part);
  float* const part = PIECE ? p.part : parts ? e.part + (size_t)tz * gy * RN * e.ldp : nullptr;
  const int on = PIECE ? n0 : 0, om = PIECE ? m0 : s.m0;    // its first row and column
  // whether all of the tile's rows and features exist
  const int fw = MODE == UP ? mt / 2 : mt;
  const bool full = (MODE == UP || MODE == DH) && n0 + RN <= e.T &&
                    (MODE == UP ? (m0 + RM) / 2 : m0 + RM) <= e.F;
  // scales of the lane's columns of codes
  float sm[8], sm1[8];
  if constexpr (sizeof(E) == 1) {
    if constexpr (MODE == UP) {
      const int f = fw + 8 * (lane % (2 * WM));
      get(e.sm + f, sm, e.F - f);
      get(e.sm1 + f, sm1, e.F - f);
    } else if (!parts) {
      const int m = mt + 8 * (lane % (RL / 8));
      get(e.sm + m, sm, e.mout - m);
    }
  }
  // the sums of 32 rows to the wave's own region, whose LDS operations stay in order
  auto stage = [&](int b) {
#pragma unroll
    for (int a = 0; a < WM; ++a)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        f32x4 v;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if constexpr (sizeof(E) == 1) v[j] = __int_as_float(acc[a][b][4 * g + j]);
          else v[j] = acc[a][b][4 * g + j];
        }
        *(f32x4*)(mine + li * RL + 4 * ((8 * a + 2 * g + h) ^ (li & (RL / 4 - 1)))) = v;
      }
    staged_fence();
  };
  if constexpr (MODE != DH) __syncthreads();     // every wave is done with the operand stages
  if constexpr (MODE == UP) {
#pragma unroll
    for (int b = 0; b < WN; ++b) {
      stage(b);
      if (full) up_rows<E, WM, ACT, true>(mine, lane, e, nt + 32 * b, fw, sm, sm1);
      else up_rows<E, WM, ACT, false>(mine, lane, e, nt + 32 * b, fw, sm, sm1);
      staged_fence();
    }
  } else if constexpr (MODE == DH) {
    if (full && e.keep == KEEP_CODES) {
      dh_full<E, true, WM, WN, ACT>(mine, lane, e, nt, mt, stage);
    } else if (full) {
      dh_full<E, false, WM, WN, ACT>(mine, lane, e, nt, mt, stage);
    } else {
      __syncthreads();
#pragma unroll
      for (int b = 0; b < WN; ++b) {
        stage(b);
        dh_rows<E, WM, ACT>(mine, lane, e, nt + 32 * b, mt, s.N);
        staged_fence();
      }
    }
  } else {
#pragma unroll
    for (int b = 0; b < WN; ++b) {
      stage(b);
      const int nb = nt + 32 * b;
      if (parts) {
        store_part<float, RL>(mine, lane, part, PIECE ? RM : e.ldp, nb - on, s.N - on, mt - om,
                              s.M - om, 0);
      } else if constexpr (sizeof(E) == 1) {
        scaled_part<O, RL>(mine, lane, e, nb, mt, sm);
      } else {
        // (32 rows are on one side of n1, a multiple of 64)
        const bool second = nb >= e.n1;
        store_part<O, RL>(mine, lane, (O*)(second ? e.out1 : e.out), second ? e.ldo1 : e.ldo,
                          second ? nb - e.n1 : nb, e.nout, mt, e.mout, e.accumulate);
      }
      staged_fence();
    }
  }
}

}  // namespace
}  // namespace hfk


// Kernels of a product: big: 256 x 256 tiles, 8 waves of 128 x 64; n64: 128 x 64, 4
// waves of 64 x 32, with three K blocks on their way, for few rows; else 128 x 128, 4
// waves of 64 x 64
// (a launch's workgroups are a line: the order of tiles is the kernel's)
#define HF_GGEMM_WIDE(NAME, E, O, MODE, ACT)                                           \
  extern "C" __global__ __launch_bounds__(512, 1) void NAME##_big(GGemm s, GEpi e) {   \
    ggemm_body<E, O, MODE, ACT, 4, 2, 2, 4, 2>(s, e, blockIdx.x);                      \
  }                                                                                    \
  extern "C" __global__ __launch_bounds__(256, 2) void NAME(GGemm s, GEpi e) {         \
    ggemm_body<E, O, MODE, ACT, 2, 2, 2, 2, 2>(s, e, blockIdx.x);                      \
  }
#define HF_GGEMM(NAME, E, O, MODE, ACT)                                                \
  HF_GGEMM_WIDE(NAME, E, O, MODE, ACT)                                                 \
  extern "C" __global__ __launch_bounds__(256, 2) void NAME##_n64(GGemm s, GEpi e) {   \
    ggemm_body<E, O, MODE, ACT, 2, 1, 2, 2, 3>(s, e, blockIdx.x);                                  \
  }
// and n32: 128 x 32, a wave having 32 of the matrix's rows, with four K blocks on their way
#define HF_GGEMM_FEW(NAME, E, O, MODE, ACT)                                            \
  HF_GGEMM(NAME, E, O, MODE, ACT)                                                      \
  extern "C" __global__ __launch_bounds__(256, 2) void NAME##_n32(GGemm s, GEpi e) {   \
    ggemm_body<E, O, MODE, ACT, 1, 1, 4, 1, 4>(s, e, blockIdx.x);                                  \
  }
#define HF_GK(NAME) {NAME, NAME##_big, NAME##_n64}
#define HF_GK_FEW(NAME) {NAME, NAME##_big, NAME##_n64, NAME##_n32}
// The kernels with an activation, a source file for each: "up" by type, "dh" by type
#define HF_GATED_ACT(SUF, ACT)                                                         \
  namespace hfk {                                                                      \
  HF_GGEMM(hf_gated_up_f32_##SUF, float, float, UP, ACT)                               \
  HF_GGEMM(hf_gated_up_bf16_##SUF, bf16_t, bf16_t, UP, ACT)                            \
  HF_GGEMM(hf_gated_up_codes_##SUF, int8_t, float, UP, ACT)                            \
  HF_GGEMM_FEW(hf_gated_dh_f32_##SUF, float, float, DH, ACT)                           \
  HF_GGEMM_FEW(hf_gated_dh_bf16_##SUF, bf16_t, bf16_t, DH, ACT)                        \
  extern const GActKernels gated_##SUF = {                                             \
      {HF_GK(hf_gated_up_f32_##SUF), HF_GK(hf_gated_up_bf16_##SUF),                    \
       HF_GK(hf_gated_up_codes_##SUF)},                                                \
      {HF_GK_FEW(hf_gated_dh_f32_##SUF), HF_GK_FEW(hf_gated_dh_bf16_##SUF)}};                  \
  }  /* namespace hfk */
