// The GEMMs of the softmax head over a large vocabulary.  With X the counted
// rows (T x D), W the vocabulary matrix (V x D) and tau the temperature:
//   logits     z = X W^T / tau, of a piece of the vocabulary; per row and 128
//              (small tiles: 64) columns the maximum and the sum of
//              exp(z - max), from which the log-sum-exp over the whole
//              vocabulary is joined.  What is kept of a piece is z itself
//              (fp32), or exp(z - max) in fp16 (bf16): 11 bits where delta
//              has 8 down to 2^-29 of the largest of the 128 (scaled by
//              2^15), in a third of the bytes of z and delta
//   p          exp(z - lse), recomputed piece by piece
//   dX         delta W, delta = p - q (q the targets), summed over the pieces
//   dW         delta^T X, whole for each piece
// 2 T V D operations each: bound by the matrix cores but for few rows, where
// reading W bounds them.
//
// C(m, n) = sum_k A(m, k) B(n, k) with m the dimension that is contiguous in
// the output: the vocabulary for logits, the width for the gradients.  A lane
// of a 32 x 32 MFMA holds one n and 16 values of m, so the maximum and the sum
// over the vocabulary run within a lane, and outputs leave as 4 consecutive
// values.
//
// No operand is transposed in memory.  A K-contiguous operand is kept in LDS
// as [row][k] and read 16 bytes a lane; one whose rows are k is kept as
// [k][row], and bf16 fragments are transposed on the way out of LDS
// (ds_read_b64_tr_b16: 16 lanes read 4 rows of 16 and get 4 values of k each),
// fp32 ones read value by value.  LDS tiles are filled by direct loads, with
// the 16-byte chunks of a row XOR-swizzled by the row so that the lanes that
// LDS serves together fall into distinct banks:
//   [row][k], 128-byte rows: chunk ^ (row / 2) % 8
//   [k][row], bf16: 64-byte runs of 4 consecutive k: chunk ^ 4 (k % 4)
//   [k][row], fp32: 128-byte runs of k and k + 4:    chunk ^ 8 (k / 4 % 2)
// K advances BK at a time through S stages, each refilled S blocks ahead once
// every wave has its last fragments in registers.  The fragment reads of the
// next step and the direct loads of the stage just freed are issued one by one
// between the MFMAs, which then run on through the change of stage: issued
// together ahead of them, they left the matrix cores idle 30% of the time
// (8,192 rows x 32,768 x 4,096 in bf16: logits 1,830 -> 1,680 us, dX 1,980 ->
// 1,730, dW 2,050 -> 1,840; fp32 16,384 x 2,048 x 2,048: 1,230 -> 975 us).
#include <type_traits>

#include "lds_dma.h"
#include "vocab_internal.h"

namespace hfk {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ uint32_t f2bf(float f) {
  return __builtin_bit_cast(uint16_t, (__bf16)f);
}
__device__ __forceinline__ float bf2f(uint32_t h) { return __uint_as_float(h << 16); }

// fragment of one step for one 32-row block: 8 consecutive k per half-wave
// (bf16, one MFMA) or 4 (fp32, four MFMAs)
template <class E>
struct FragT;
template <>
struct FragT<bf16_t> { typedef bf16x8 T; };
template <>
struct FragT<float> { typedef f32x4 T; };

template <class E, bool KC, int ROWS, int BK, int NW>
struct Tile {
  typedef typename FragT<E>::T Frag;
  static constexpr int EPC = 16 / (int)sizeof(E);     // elements per chunk
  static constexpr int CH = KC ? BK / EPC : ROWS / EPC;
  static constexpr int SIZE = ROWS * BK;
  static constexpr int INSTR = SIZE / EPC / 64 / NW;
  static_assert(SIZE % (EPC * 64 * NW) == 0, "tile does not split over the waves");
  static_assert(BK * sizeof(E) <= 128 && (KC || ROWS * sizeof(E) >= 256), "swizzles");

  __device__ static __forceinline__ int swz(int r) {
    if (KC) return (r / (256 / (BK * (int)sizeof(E)))) % CH;
    return sizeof(E) == 2 ? (r & 3) << 2 : ((r >> 2) & 1) << 3;
  }
  // the LDS row (of rows, or of k) and the global chunk that `lane` of `wave`
  // fetches with its direct load j
  __device__ static __forceinline__ void src(int wave, int lane, int j, int& row, int& ch) {
    const int P = (wave * INSTR + j) * 64 + lane;
    row = P / CH;
    ch = (P % CH) ^ swz(row);
  }
  __device__ static __forceinline__ int dst(int wave, int j) {
    return (wave * INSTR + j) * 64 * EPC;
  }
  // step q of the 32-row block at row0, for lane (li, h)
  __device__ static __forceinline__ Frag frag(const E* s, int row0, int lane, int q) {
    const int li = lane & 31, h = lane >> 5;
    if constexpr (KC) {
      const int row = row0 + li;
      return *(const Frag*)(s + row * BK + (((2 * q + h) ^ swz(row)) * EPC));
    } else if constexpr (sizeof(E) == 2) {
      const int l = lane & 15, col = row0 + (lane & 16) + 4 * (l & 3);
      s16x4 v[2];
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const int k = 16 * q + 8 * h + 4 * r + (l >> 2);
        const E* p = s + k * ROWS + (((col >> 3) ^ swz(k)) << 3) + (col & 7);
        v[r] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) s16x4*)p);
      }
      return __builtin_bit_cast(
          bf16x8, __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
      const int col = row0 + li;
      Frag f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int k = 8 * q + 4 * h + j;
        f[j] = s[k * ROWS + (((col >> 2) ^ swz(k)) << 2) + (col & 3)];
      }
      return f;
    }
  }
};

// product j of a step: one with bf16, four with fp32 (all blocks take their
// j-th one after the other, so that no MFMA waits for the one before it)
__device__ __forceinline__ f32x16 mma1(bf16x8 a, bf16x8 b, f32x16 c, int) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma1(f32x4 a, f32x4 b, f32x16 c, int j) {
  return __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], c, 0, 0, 0);
}

// exp, to the last bits where the type keeps them
template <class E>
__device__ __forceinline__ float exp_of(float x) {
  return sizeof(E) == 4 ? expf(x) : __expf(x);
}
__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ float load1(const bf16_t* p) { return bf2f(*p); }
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }
__device__ __forceinline__ float load1(const _Float16* p) { return (float)*p; }
__device__ __forceinline__ void store1(bf16_t* p, float v) { *p = (bf16_t)f2bf(v); }
__device__ __forceinline__ void store1(_Float16* p, float v) { *p = (_Float16)v; }
// whole 16-byte chunks, of any alignment
__device__ __forceinline__ void add_chunk(const float* p, float (&v)[4]) {
  f32x4 o;
  __builtin_memcpy(&o, p, 16);
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] += o[j];
}
__device__ __forceinline__ void add_chunk(const bf16_t* p, float (&v)[8]) {
  u32x4 o;
  __builtin_memcpy(&o, p, 16);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    v[2 * j] += bf2f(o[j] & 0xffffu);
    v[2 * j + 1] += bf2f(o[j] >> 16);
  }
}
__device__ __forceinline__ void add_chunk(const _Float16*, float (&)[8]) {}
// STREAM: past the caches
template <bool STREAM>
__device__ __forceinline__ void put16(void* p, u32x4 w) {
  typedef u32x4 __attribute__((aligned(2))) loose;
  if (STREAM) __builtin_nontemporal_store(w, (loose*)p);
  else *(loose*)p = w;
}
template <bool STREAM>
__device__ __forceinline__ void store_chunk(_Float16* p, const float (&v)[8]) {
  typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
  f16x8 w;
#pragma unroll
  for (int j = 0; j < 8; ++j) w[j] = (_Float16)v[j];
  put16<STREAM>(p, __builtin_bit_cast(u32x4, w));
}
template <bool STREAM>
__device__ __forceinline__ void store_chunk(float* p, const float (&v)[4]) {
  put16<STREAM>(p, __builtin_bit_cast(u32x4, f32x4{v[0], v[1], v[2], v[3]}));
}
template <bool STREAM>
__device__ __forceinline__ void store_chunk(bf16_t* p, const float (&v)[8]) {
  u32x4 w;
#pragma unroll
  for (int j = 0; j < 4; ++j) w[j] = f2bf(v[2 * j]) | f2bf(v[2 * j + 1]) << 16;
  put16<STREAM>(p, w);
}

// One 32-row part (rows n0 .. n0 + 31) of a wave's tile to memory: RL columns
// from m0, up to row Np and column Mp, from the wave's LDS region s, where
// row r's 16-byte chunk c is at c ^ r % (RL / 4).  Through LDS, a store
// instruction covers whole 256- or 512-byte runs of rows instead of 16-byte
// pieces of 32 rows.
// add: += what is there; idx: the row of out for each row.  STREAM: for much
// that nothing reads soon (dW), so that it does not take the place of what is read
// (5 rows, 32,000 x 1,024 of bf16: 18.0 -> 16.2 us; 120 rows, 50,257 x 2,048:
// 100 -> 88).
template <class O, int RL, bool STREAM = false>
__device__ __forceinline__ void store_part(const float* s, int lane, O* out, long long ldo,
                                           int n0, int Np, int m0, int Mp, int add,
                                           const int* idx = nullptr) {
  constexpr int OPC = 16 / (int)sizeof(O), CPR = RL / OPC, Q = RL / 4;
#pragma unroll
  for (int i = 0; i < 32 * CPR / 64; ++i) {
    const int r = (lane + 64 * i) / CPR, c = (lane + 64 * i) % CPR;
    const int n = n0 + r, m = m0 + OPC * c;
    if (n >= Np || m >= Mp) continue;
    float v[OPC];
#pragma unroll
    for (int k = 0; k < OPC / 4; ++k) {
      const f32x4 w = *(const f32x4*)(s + r * RL + 4 * ((c * (OPC / 4) + k) ^ (r & (Q - 1))));
#pragma unroll
      for (int j = 0; j < 4; ++j) v[4 * k + j] = w[j];
    }
    O* p = out + (size_t)(idx ? idx[n] : n) * ldo + m;
    if (m + OPC <= Mp) {
      if (add) add_chunk(p, v);
      store_chunk<STREAM>(p, v);
    } else {
#pragma unroll
      for (int j = 0; j < OPC; ++j)
        if (m + j < Mp) store1(p + j, add ? v[j] + load1(p + j) : v[j]);
    }
  }
}

// ----------------------------------------------------------------- epilogues
enum { E_LOGITS, E_EXPS, E_PROBS, E_PART, E_OUT, E_STREAM, E_ROWS };

// The tile (tm, tn) and split this workgroup computes, of gy tiles of n that
// have rows and gz splits; false: none.  Consecutive workgroups go to the 8
// XCDs in turn; each XCD gets a contiguous eighth of the logical order, which
// walks groups of 8 tiles of n, m by m, so that the workgroups resident on an
// XCD share their operand panels in its L2.  Tiles without rows take no place
// in the order (2,251 of 3,001 rows counted, 50,257 x 1,024: 301 -> 222 us).
__device__ __forceinline__ bool tile_of(int gy, int gz, int& tm, int& tn, int& tz) {
  const int gx = gridDim.x;
  const int T = gx * gy * gz;
  const int L = blockIdx.x + gx * (blockIdx.y + gridDim.y * blockIdx.z);
  if (L >= T) return false;
  // XCD x's share: T / 8 workgroups, one more for the first T % 8
  const int x = L % 8, q = T / 8, r8 = T % 8;
  const int Lg = x * q + min(x, r8) + L / 8;
  tz = Lg / (gx * gy);
  const int r = Lg % (gx * gy);
  constexpr int G = 8;
  const int g = r / (G * gx);
  const int first = g * G;
  const int rows = min(G, gy - first);
  const int w = r - g * G * gx;
  tn = first + w % rows;
  tm = w / rows;
  return true;
}

template <class E, int EPI, bool AKC, bool BKC, int WM, int WN, int GM, int GN, int S, int KB>
__device__ __forceinline__ void vgemm_body(const VGemm& s, const VEpi& e) {
  constexpr int BK = KB / (int)sizeof(E);
  constexpr int NW = GM * GN;
  constexpr int RM = 32 * WM * GM, RN = 32 * WN * GN;
  using TA = Tile<E, AKC, RM, BK, NW>;
  using TB = Tile<E, BKC, RN, BK, NW>;
  constexpr int EPC = TA::EPC;
  constexpr int STAGE = TA::SIZE + TB::SIZE;
  constexpr int LPB = TA::INSTR + TB::INSTR;
  __shared__ __attribute__((aligned(16))) E lds[S * STAGE];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / GN, wn = wave % GN;
  const int li = lane & 31, h = lane >> 5;
  const int nrow = s.st->n;
  const int N = s.dyn == 1 ? nrow : s.N;
  const int K = s.dyn == 2 ? (nrow + BK - 1) & ~(BK - 1) : s.K;
  const int gy = (N + RN - 1) / RN;
  const int splits = splits_of(s.splits, s.smax, gridDim.y, gy);
  int tm, tn, tz;
  if (!tile_of(gy, splits, tm, tn, tz)) return;
  const int m0 = tm * RM, n0 = tn * RN;
  // rows that all count are read where they are, not packed
  const bool whole = s.X && nrow == s.T;
  constexpr bool XA = !BKC;              // dW: X is A; logits: X is B
  const int alim = XA && whole ? s.T : s.alim;
  const int blim = !XA && whole ? s.T : s.blim;

  const int nvb = (K + BK - 1) / BK;
  int vb0 = 0, nblk = nvb;
  if (splits > 1) {
    const int per = (nvb + splits - 1) / splits;
    vb0 = min(tz * per, nvb);
    nblk = min(nvb, vb0 + per) - vb0;
  }

  f32x16 acc[WM][WN];
#pragma unroll
  for (int a = 0; a < WM; ++a)
#pragma unroll
    for (int b = 0; b < WN; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[a][b][r] = 0.0f;

  // fp32 logits: the sum of the K blocks before these SUM_COLS columns (see there)
  constexpr bool PARTS = (EPI == E_LOGITS || EPI == E_PROBS) && sizeof(E) == 4 && WM * WN < 8;
  static_assert(SUM_COLS % BK == 0, "K blocks of a sum");
  f32x16 before[PARTS ? WM : 1][PARTS ? WN : 1];
  if constexpr (PARTS) {
#pragma unroll
    for (int a = 0; a < WM; ++a)
#pragma unroll
      for (int b = 0; b < WN; ++b) before[a][b] = acc[a][b];
  }
  auto add_up = [&]() {
    if constexpr (PARTS) {
#pragma unroll
      for (int a = 0; a < WM; ++a)
#pragma unroll
        for (int b = 0; b < WN; ++b)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            before[a][b][r] += acc[a][b][r];
            acc[a][b][r] = 0.0f;
          }
    }
  };

  // Element offsets of the lane's direct loads from the tile's origin.  Rows
  // of a K-contiguous operand past its last one read that one; chunks of a
  // [k][m] operand past its padded width read the last chunk (both feed
  // outputs that are not stored).
  const long long lda = XA && whole ? s.ldx : s.lda, ldb = !XA && whole ? s.ldx : s.ldb;
  uint32_t offa[TA::INSTR], offb[TB::INSTR];
#pragma unroll
  for (int j = 0; j < TA::INSTR; ++j) {
    int row, ch;
    TA::src(wave, lane, j, row, ch);
    if (AKC) offa[j] = (uint32_t)((min(m0 + row, alim - 1) - m0) * lda) + EPC * ch;
    else offa[j] = (uint32_t)(row * lda) + min(EPC * ch, (int)(s.M - 1 - m0) / EPC * EPC);
  }
#pragma unroll
  for (int j = 0; j < TB::INSTR; ++j) {
    int row, ch;
    TB::src(wave, lane, j, row, ch);
    if (BKC) offb[j] = (uint32_t)((min(n0 + row, blim - 1) - n0) * ldb) + EPC * ch;
    else offb[j] = (uint32_t)(row * ldb) + EPC * ch;
  }
  const E* const A0 = (const E*)(XA && whole ? s.X : s.A) + (AKC ? (size_t)m0 * lda : (size_t)m0);
  const E* const B0 = (const E*)(!XA && whole ? s.X : s.B) + (BKC ? (size_t)n0 * ldb : (size_t)n0);
  const uint32_t lds0 = lds_address(lds);
  // direct load j of K block vb into stage st (A's, then B's)
  auto issue1 = [&](int vb, int st, int j) {
    const int k0 = vb * BK;
    const uint32_t base = lds0 + (uint32_t)sizeof(E) * (uint32_t)(st * STAGE);
    if (j < TA::INSTR) {
      const E* a = A0 + (AKC ? (size_t)k0 : (size_t)k0 * lda);
      // rows of k past the last one read the last one, against zeros of B
      long long o = offa[j];
      if (!AKC && k0 + BK > alim) {
        int row, ch;
        TA::src(wave, lane, j, row, ch);
        o -= max(0, k0 + row - (alim - 1)) * lda;
      }
      dma16_at(a + o, base + (uint32_t)sizeof(E) * TA::dst(wave, j));
    } else {
      const E* b = B0 + (BKC ? (size_t)k0 : (size_t)k0 * ldb);
      dma16_at(b + offb[j - TA::INSTR],
               base + (uint32_t)sizeof(E) * (TA::SIZE + TB::dst(wave, j - TA::INSTR)));
    }
  };
  auto issue = [&](int vb, int st) {
#pragma unroll
    for (int j = 0; j < LPB; ++j) issue1(vb, st, j);
  };

  struct Frags {
    typename TA::Frag a[WM];
    typename TB::Frag b[WN];
  };
  constexpr int NF = WM + WN;
  auto fetch1 = [&](Frags& f, int st, int q, int i) {
    const E* la = lds + st * STAGE;
    const E* lb = la + TA::SIZE;
    if (i < WN) f.b[i] = TB::frag(lb, wn * 32 * WN + 32 * i, lane, q);
    else f.a[i - WN] = TA::frag(la, wm * 32 * WM + 32 * (i - WN), lane, q);
  };
  auto fetch = [&](Frags& f, int st, int q) {
#pragma unroll
    for (int i = 0; i < NF; ++i) fetch1(f, st, q, i);
  };
  // the MFMAs of a step; side(i) after the i-th of them, which issues its share
  // of the next step's fragment reads (FT) and direct loads (AT)
  constexpr int NJ = (int)sizeof(E) * (int)sizeof(E) / 4, NM = NJ * WM * WN;
  constexpr int FT = (NF + NM - 1) / NM, AT = (LPB + NM - 1) / NM;
  constexpr int PER = NM / LPB > 0 ? NM / LPB : 1;      // MFMAs per direct load
  auto mma = [&](const Frags& f, auto side) {
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int a = 0; a < WM; ++a)
#pragma unroll
        for (int b = 0; b < WN; ++b) {
          acc[a][b] = mma1(f.a[a], f.b[b], acc[a][b], j);
          side((j * WM + a) * WN + b);
          __builtin_amdgcn_sched_barrier(0);
        }
  };

  constexpr int NQ = KB / 32;      // steps per K block
  static_assert(NQ % 2 == 0 && (S - 1) * LPB < 64, "pipeline depth");
  Frags fa, fb;
#pragma unroll
  for (int i = 0; i < S; ++i)
    if (i < nblk) issue(vb0 + i, i);
  // the rows' labels, for the epilogue: behind the first stages, which the waits
  // below are for (4,096 rows, 50,257 x 768: a loss 314 -> 317 us, where a pass of
  // its own over the labels' rows of W took 2 in hf_vocab_row_loss; ahead of the
  // stages 324 -> 329)
  constexpr bool STATS = EPI == E_LOGITS || EPI == E_EXPS;
  int lab[WN];
  if constexpr (STATS) {
#pragma unroll
    for (int b = 0; b < WN; ++b) {
      const int n = n0 + wn * 32 * WN + 32 * b + li;
      lab[b] = e.lab && n < N ? e.lab[n] : -1;
    }
  }
  if (nblk > 0) {
    if (nblk >= S) wait_vm<(S - 1) * LPB>();
    else wait_vm<0>();
    stage_barrier();
    fetch(fa, 0, 0);
  }
  for (int it = 0; it < nblk; ++it) {
    const int st = it % S;
#pragma unroll
    for (int q = 0; q + 1 < NQ; ++q) {
      Frags& nx = (q & 1) ? fa : fb;
      mma((q & 1) ? fb : fa, [&](int i) {
#pragma unroll
        for (int x = 0; x < FT; ++x)
          if (i * FT + x < NF) fetch1(nx, st, q + 1, i * FT + x);
      });
    }
    // this wave's loads of block it + 1 have landed once at most
    // min(S - 2, nblk - 2 - it) later blocks are pending
    wait_vm<(S - 2) * LPB>();
    if (S > 2 && nblk - 2 - it < S - 2) wait_vm<0>();
    stage_barrier();       // every wave's loads landed; stage st is free
    const bool more = it + S < nblk;
    const int vb = vb0 + it + S;
    mma(fb, [&](int i) {
      // (past the last block: a read of a stage that nobody writes, unused)
#pragma unroll
      for (int x = 0; x < FT; ++x)
        if (i * FT + x < NF) fetch1(fa, (it + 1) % S, 0, i * FT + x);
      if (i % PER == 0 && i / PER * AT < LPB && more) {
#pragma unroll
        for (int x = 0; x < AT; ++x)
          if (i / PER * AT + x < LPB) issue1(vb, st, i / PER * AT + x);
      }
    });
    if ((it + 1) % (SUM_COLS / BK) == 0) add_up();
  }
  if constexpr (PARTS) {
#pragma unroll
    for (int a = 0; a < WM; ++a)
#pragma unroll
      for (int b = 0; b < WN; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[a][b][r] = before[a][b][r] + acc[a][b][r];
  }

  // Lane (li, h), register r of block (a, b) holds n = 32 b + li and
  // m = 32 a + 8 (r / 4) + 4 h + r % 4 of the wave's part of the tile.
  const int mt = m0 + wm * 32 * WM, nt = n0 + wn * 32 * WN;
  const int mw = mt + 4 * h;
  constexpr int RL = 32 * WM;
  static_assert(NW * 32 * RL * 4 <= S * STAGE * (int)sizeof(E), "staging exceeds the stages");
  float* const mine = (float*)lds + wave * 32 * RL;
  if constexpr (STATS) {
    // row statistics of the wave's columns: within the lane, then the two
    // halves of the wave.  exp(z - max) = exp2((acc - max) c): an argument off
    // by 2^-24 of its size weighs exp of minus that size, so exp2 itself is
    // exact enough for fp32
    const float c2 = e.zscale * 1.44269504f;
    const bool full = m0 + RM <= s.M;
    // (a wait for one of them further down would be a wait for the stores before
    // it too)
#pragma unroll
    for (int b = 0; b < WN; ++b) asm volatile("" : "+v"(lab[b]));
#pragma unroll
    for (int b = 0; b < WN; ++b) {
      if (!full) {
#pragma unroll
        for (int a = 0; a < WM; ++a)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (mw + 32 * a + 8 * (r >> 2) + (r & 3) >= s.M) acc[a][b][r] = -INFINITY;
      }
      // The label's logit, the very number that is in the sums: of a word with
      // nearly all the probability a logit summed in another order is off by
      // more than what is left for the others.  Few waves have one (128 of
      // 50,000 columns, 32 rows: 8%).
      if (e.lab) {
        const int d = lab[b] - e.v0 - mt;
        const bool here = lab[b] >= 0 && d >= 0 && d < RL && ((d >> 2) & 1) == h;
        if (__ballot(here)) {
          float x = 0.0f;
#pragma unroll
          for (int a = 0; a < WM; ++a)
#pragma unroll
            for (int r = 0; r < 16; ++r)
              if (4 * (d >> 3) + (d & 3) == 16 * a + r) x = acc[a][b][r];
          if (here) e.zt[nt + 32 * b + li] = x * e.zscale;
        }
      }
      float mx = -INFINITY;
#pragma unroll
      for (int a = 0; a < WM; ++a)
#pragma unroll
        for (int r = 0; r < 16; ++r) mx = fmaxf(mx, acc[a][b][r]);
      mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
      // nothing but -inf: exp(-inf - 0) = 0, where -inf - -inf is no number
      const float at = mx == -INFINITY ? 0.0f : mx;
      float sum = 0.0f;
#pragma unroll
      for (int a = 0; a < WM; ++a)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float x = __builtin_amdgcn_exp2f((acc[a][b][r] - at) * c2);
          sum += x;
          if (EPI == E_EXPS) acc[a][b][r] = x * EXP_SCALE;
        }
      sum += __shfl_xor(sum, 32, 64);
      const int n = nt + 32 * b + li;
      if (h == 0 && n < N && mt < s.M)
        e.stat[(size_t)n * e.ldstat + e.tile0 + mt / RL] = float2{mx * e.zscale, sum};
    }
    if (EPI == E_LOGITS && !e.z) return;
    __syncthreads();     // every wave is done with the operand stages
  } else {
    __syncthreads();     // every wave is done with the operand stages
  }
  // columns and rows of p are written up to whole K blocks of the products
  // that read them: zeros past the piece and past the last row
  const int Mp = EPI == E_PROBS || STATS ? (s.M + VPAD - 1) & ~(VPAD - 1) : s.M;
  const int Np = EPI == E_PROBS ? (N + VPAD - 1) & ~(VPAD - 1) : N;
  constexpr bool FINAL = EPI == E_OUT || EPI == E_STREAM || EPI == E_ROWS;
  const bool parts = EPI == E_PART || (EPI == E_ROWS && splits > 1);
  const float scale = FINAL && !parts ? s.st->gscale : 1.0f;
  float* const part = e.part + (size_t)tz * gy * RN * e.ldp;
#pragma unroll
  for (int b = 0; b < WN; ++b) {
    const int n = nt + 32 * b + li;
    const float lse = EPI == E_PROBS && n < N ? e.lse[n] : 0.0f;
#pragma unroll
    for (int a = 0; a < WM; ++a)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        f32x4 v;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float c = acc[a][b][4 * g + j];
          if (EPI == E_PROBS)
            v[j] = n < N && mw + 32 * a + 8 * g + j < s.M ? exp_of<E>(c * e.zscale - lse) : 0.0f;
          else v[j] = FINAL ? c * scale : EPI == E_LOGITS ? c * e.zscale : c;
        }
        *(f32x4*)(mine + li * RL + 4 * ((8 * a + 2 * g + h) ^ (li & (RL / 4 - 1)))) = v;
      }
    // the wave's own region, and its LDS operations stay in order
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    const int nb = nt + 32 * b;
    if constexpr (EPI == E_LOGITS)
      store_part<float, RL>(mine, lane, e.z, e.ldz, nb, Np, mt, Mp, 0);
    else if constexpr (EPI == E_EXPS)
      store_part<_Float16, RL>(mine, lane, (_Float16*)e.pt, e.ldz, nb, Np, mt, Mp, 0);
    else if constexpr (EPI == E_PROBS)
      store_part<E, RL>(mine, lane, (E*)e.d, e.ldd, nb, Np, mt, Mp, 0);
    else if constexpr (EPI == E_OUT || EPI == E_STREAM)
      store_part<E, RL, EPI == E_STREAM>(mine, lane, (E*)e.out, e.ldo, nb, Np, mt, Mp,
                                         e.accumulate);
    else if (parts)
      store_part<float, RL>(mine, lane, part, e.ldp, nb, Np, mt, Mp, e.add);
    else if constexpr (EPI == E_ROWS)
      store_part<E, RL>(mine, lane, (E*)e.out, e.ldo, nb, Np, mt, Mp, 0, e.idx);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
}

}  // namespace

// big: 256 x 256 tiles, 8 waves of 128 x 64; else 128 x 128, 4 waves of 64 x 64
#define HF_VGEMM(NAME, EPI, AKC, BKC)                                                  \
  extern "C" __global__ __launch_bounds__(512, 1) void NAME##_bf16_big(VGemm s, VEpi e) { \
    vgemm_body<bf16_t, EPI, AKC, BKC, 4, 2, 2, 4, 2, 128>(s, e);                       \
  }                                                                                    \
  extern "C" __global__ __launch_bounds__(256, 2) void NAME##_bf16(VGemm s, VEpi e) {  \
    vgemm_body<bf16_t, EPI, AKC, BKC, 2, 2, 2, 2, 2, 128>(s, e);                       \
  }                                                                                    \
  extern "C" __global__ __launch_bounds__(512, 1) void NAME##_f32_big(VGemm s, VEpi e) {  \
    vgemm_body<float, EPI, AKC, BKC, 4, 2, 2, 4, 2, 128>(s, e);                        \
  }                                                                                    \
  extern "C" __global__ __launch_bounds__(256, 2) void NAME##_f32(VGemm s, VEpi e) {   \
    vgemm_body<float, EPI, AKC, BKC, 2, 2, 2, 2, 2, 128>(s, e);                        \
  }
// up to 1,024 rows of X: 128 x 64 and 128 x 32 tiles, a wave having 32 of W's rows, with
// three K blocks of W on their way; bound by the reads of W
#define HF_VGEMM_FEW(NAME, EPI, AKC, BKC)                                              \
  extern "C" __global__ __launch_bounds__(256, 2) void NAME##_bf16_n64(VGemm s, VEpi e) { \
    vgemm_body<bf16_t, EPI, AKC, BKC, 1, 2, 4, 1, 3, 128>(s, e);                       \
  }                                                                                    \
  extern "C" __global__ __launch_bounds__(256, 2) void NAME##_bf16_n32(VGemm s, VEpi e) { \
    vgemm_body<bf16_t, EPI, AKC, BKC, 1, 1, 4, 1, 4, 128>(s, e);                       \
  }                                                                                    \
  extern "C" __global__ __launch_bounds__(256, 2) void NAME##_f32_n64(VGemm s, VEpi e) {  \
    vgemm_body<float, EPI, AKC, BKC, 1, 2, 4, 1, 3, 128>(s, e);                        \
  }                                                                                    \
  extern "C" __global__ __launch_bounds__(256, 2) void NAME##_f32_n32(VGemm s, VEpi e) {  \
    vgemm_body<float, EPI, AKC, BKC, 1, 1, 4, 1, 4, 128>(s, e);                        \
  }
HF_VGEMM_FEW(hf_vocab_logits, E_LOGITS, true, true)
HF_VGEMM_FEW(hf_vocab_dx, E_PART, false, true)
HF_VGEMM(hf_vocab_logits, E_LOGITS, true, true)
extern "C" __global__ __launch_bounds__(512, 1) void hf_vocab_exps_bf16_big(VGemm s, VEpi e) {
  vgemm_body<bf16_t, E_EXPS, true, true, 4, 2, 2, 4, 2, 128>(s, e);
}
extern "C" __global__ __launch_bounds__(256, 2) void hf_vocab_exps_bf16(VGemm s, VEpi e) {
  vgemm_body<bf16_t, E_EXPS, true, true, 2, 2, 2, 2, 2, 128>(s, e);
}
HF_VGEMM(hf_vocab_probs, E_PROBS, true, true)
HF_VGEMM(hf_vocab_dx, E_PART, false, true)
HF_VGEMM(hf_vocab_dx_out, E_ROWS, false, true)
HF_VGEMM(hf_vocab_dw, E_OUT, false, false)
HF_VGEMM(hf_vocab_dw_part, E_PART, false, false)
// dW of few rows: bound by the stores of its output, so three workgroups per
// compute unit, with half the K block, cover each other's latency better (5
// rows x 32,000 x 1,024: 21 -> 17.6 us)
#define HF_VGEMM_THIN(SUF, E, EPI)                                                        \
  extern "C" __global__ __launch_bounds__(256, 3) void hf_vocab_dw_##SUF(VGemm s, VEpi e) { \
    vgemm_body<E, EPI, false, false, 2, 2, 2, 2, 2, 64>(s, e);                            \
  }
HF_VGEMM_THIN(f32_thin, float, E_OUT)
HF_VGEMM_THIN(bf16_thin, bf16_t, E_OUT)
HF_VGEMM_THIN(f32_thin_s, float, E_STREAM)
HF_VGEMM_THIN(bf16_thin_s, bf16_t, E_STREAM)

// ------------------------------------------------------------- launchers
namespace {
typedef void (*VK)(VGemm, VEpi);
// kernels of a product by type and tile (VT_* of VGemm::tile)
typedef VK Kernels[2][4];
void launch(const Launch& L, const char* name, const Kernels& k, int type, const VGemm& g,
            const VEpi& e) {
  if (g.M < 1 || g.N < 1) return;
  const int RM = tile_m(g.tile), RN = tile_n(g.tile);
  const dim3 grid((g.M + RM - 1) / RM, (g.N + RN - 1) / RN, g.splits);
  prof_begin(L, name);
  hipExtLaunchKernelGGL(k[type][g.tile], grid, dim3(g.tile == TILE_BIG ? 512 : 256), 0, L.stream,
                        prof_a(L), prof_b(L), 0, g, e);
  prof_end(L, name, 2.0 * g.M * (double)g.N * g.K, 0.0);
}
}  // namespace

#define HF_VK(NAME) {{NAME##_f32, NAME##_f32_big}, {NAME##_bf16, NAME##_bf16_big}}
#define HF_VK_FEW(NAME)                                               \
  {{NAME##_f32, NAME##_f32_big, NAME##_f32_n64, NAME##_f32_n32},      \
   {NAME##_bf16, NAME##_bf16_big, NAME##_bf16_n64, NAME##_bf16_n32}}
void vocab_logits(const Launch& L, int type, const VGemm& g, const VEpi& e) {
  static const Kernels k = HF_VK_FEW(hf_vocab_logits);
  static const Kernels x = {{}, {hf_vocab_exps_bf16, hf_vocab_exps_bf16_big}};
  launch(L, "hf_vocab_logits", e.pt ? x : k, type, g, e);
}
void vocab_probs(const Launch& L, int type, const VGemm& g, const VEpi& e) {
  static const Kernels k = HF_VK(hf_vocab_probs);
  launch(L, "hf_vocab_probs", k, type, g, e);
}
void vocab_dx(const Launch& L, int type, const VGemm& g, const VEpi& e) {
  static const Kernels k = HF_VK_FEW(hf_vocab_dx), o = HF_VK(hf_vocab_dx_out);
  launch(L, "hf_vocab_dx", e.out ? o : k, type, g, e);
}
void vocab_dw(const Launch& L, int type, const VGemm& g, const VEpi& e) {
  static const Kernels k = HF_VK(hf_vocab_dw), p = HF_VK(hf_vocab_dw_part);
  static const Kernels thin = {{hf_vocab_dw_f32_thin}, {hf_vocab_dw_bf16_thin}};
  static const Kernels much = {{hf_vocab_dw_f32_thin_s}, {hf_vocab_dw_bf16_thin_s}};
  launch(L, "hf_vocab_dw", g.splits > 1 ? p : !g.thin ? k : e.stream ? much : thin, type, g, e);
}

}  // namespace hfk
