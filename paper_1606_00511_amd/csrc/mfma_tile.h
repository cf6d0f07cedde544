// Tiles of the MFMA products whose operands lie as they are in memory (the
// vocabulary head's and the gated block's): direct loads into swizzled LDS,
// fragments, the order of workgroups, the K loop and the stores of a tile.
//
// C(m, n) = sum_k A(m, k) B(n, k), stored with m contiguous.  A K-contiguous
// operand is kept in LDS as [row][k] and read 16 bytes a lane; one whose rows
// are k is kept as [k][row], and bf16 fragments are transposed on the way out
// of LDS (ds_read_b64_tr_b16: 16 lanes read 4 rows of 16 and get 4 values of k
// each), fp32 ones read value by value.  LDS tiles are filled by direct loads,
// with the 16-byte chunks of a row XOR-swizzled by the row so that the lanes
// that LDS serves together fall into distinct banks:
//   [row][k], 128-byte rows: chunk ^ (row / 2) % 8
//   [k][row], bf16: 64-byte runs of 4 consecutive k: chunk ^ 4 (k % 4)
//   [k][row], fp32: 128-byte runs of k and k + 4:    chunk ^ 8 (k / 4 % 2)
#pragma once

#include "lds_dma.h"
#include "hf_internal.h"

namespace hfk {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

__device__ __forceinline__ uint32_t f2bf(float f) {
  return __builtin_bit_cast(uint16_t, (__bf16)f);
}
__device__ __forceinline__ float bf2f(uint32_t h) { return __uint_as_float(h << 16); }

// fragment of one step for one 32-row block: 16 or 8 consecutive k per half-wave
// (codes, bf16: one MFMA) or 4 (fp32, four MFMAs)
template <class E>
struct FragT;
template <>
struct FragT<bf16_t> { typedef bf16x8 T; };
template <>
struct FragT<float> { typedef f32x4 T; };
template <>
struct FragT<int8_t> { typedef i32x4 T; };
// sums of a 32 x 32 block: whole numbers of codes, which are exact
template <class E>
struct SumT { typedef f32x16 T; };
template <>
struct SumT<int8_t> { typedef i32x16 T; };

template <class E, bool KC, int ROWS, int BK, int NW>
struct Tile {
  typedef typename FragT<E>::T Frag;
  static constexpr int EPC = 16 / (int)sizeof(E);     // elements per chunk
  static constexpr int CH = KC ? BK / EPC : ROWS / EPC;
  static constexpr int SIZE = ROWS * BK, DEPTH = BK;
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

// product j of a step: one with codes or bf16, four with fp32 (all blocks take their
// j-th one after the other, so that no MFMA waits for the one before it)
__device__ __forceinline__ f32x16 mma1(bf16x8 a, bf16x8 b, f32x16 c, int) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma1(f32x4 a, f32x4 b, f32x16 c, int j) {
  return __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], c, 0, 0, 0);
}

__device__ __forceinline__ i32x16 mma1(i32x4 a, i32x4 b, i32x16 c, int) {
  return __builtin_amdgcn_mfma_i32_32x32x32_i8(a, b, c, 0, 0, 0);
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

// Tile r of gx x gy in an order that walks groups of 8 tiles of n, m by m; and its
// place in that order.
constexpr int TILE_GROUP = 8;
__device__ __forceinline__ void tile_in(int r, int gx, int gy, int& tm, int& tn) {
  const int g = r / (TILE_GROUP * gx);
  const int first = g * TILE_GROUP;
  const int rows = min(TILE_GROUP, gy - first);
  const int w = r - g * TILE_GROUP * gx;
  tn = first + w % rows;
  tm = w / rows;
}
__device__ __forceinline__ int tile_place(int tm, int tn, int gx, int gy) {
  const int first = tn / TILE_GROUP * TILE_GROUP;
  return first * gx + tm * min(TILE_GROUP, gy - first) + tn - first;
}

// The tile (tm, tn) and split this workgroup computes, of gy tiles of n that
// have rows and gz splits; false: none.  Consecutive workgroups go to the 8
// XCDs in turn; each XCD gets a contiguous eighth of the order of tile_in, so that
// the workgroups resident on an XCD share their operand panels in its L2.  Tiles without rows take no place
// in the order (2,251 of 3,001 rows counted, 50,257 x 1,024: 301 -> 222 us).
__device__ __forceinline__ bool tile_at(int L, int gx, int gy, int gz, int& tm, int& tn, int& tz) {
  const int T = gx * gy * gz;
  if (L >= T) return false;
  // XCD x's share: T / 8 workgroups, one more for the first T % 8
  const int x = L % 8, q = T / 8, r8 = T % 8;
  const int Lg = x * q + min(x, r8) + L / 8;
  tz = Lg / (gx * gy);
  tile_in(Lg % (gx * gy), gx, gy, tm, tn);
  return true;
}
__device__ __forceinline__ bool tile_of(int gy, int gz, int& tm, int& tn, int& tz) {
  return tile_at(blockIdx.x + gridDim.x * (blockIdx.y + gridDim.y * blockIdx.z), gridDim.x, gy, gz,
                 tm, tn, tz);
}

// The K loop of a workgroup's tile: acc(a, b) += the products of a wave's blocks
// over the K blocks [vb0, vb0 + nblk), in S stages of LDS.
//   issue1(vb, st, j)  direct load j of K block vb into stage st
//   fetch1(f, st, q, i)  fragment i of step q from stage st: b[0 .. WN - 1], then
//                      a.  (Passed in: with the stages' address as an argument
//                      here, two more instructions a read and 1% of a product.)
//   ahead()            loads for the epilogue, behind those of the first stages
//   block(it)          after K block it of the loop
// K advances a block at a time through S stages, each refilled S blocks ahead once
// every wave has its last fragments in registers.  The fragment reads of the
// next step and the direct loads of the stage just freed are issued one by one
// between the MFMAs, which then run on through the change of stage: issued
// together ahead of them, they left the matrix cores idle 30% of the time
// (8,192 rows x 32,768 x 4,096 in bf16: logits 1,830 -> 1,680 us, dX 1,980 ->
// 1,730, dW 2,050 -> 1,840; fp32 16,384 x 2,048 x 2,048: 1,230 -> 975 us).
template <class E, class TA, class TB, int WM, int WN>
struct FragsT {
  typename TA::Frag a[WM];
  typename TB::Frag b[WN];
};
template <class E, class TA, class TB, int WM, int WN, int S, class Acc, class Fetch1, class Issue1,
          class Ahead, class Block>
__device__ __forceinline__ void k_loop(Acc (&acc)[WM][WN], int vb0, int nblk, Fetch1 fetch1,
                                       Issue1 issue1, Ahead ahead, Block block) {
  typedef FragsT<E, TA, TB, WM, WN> Frags;
  constexpr int LPB = TA::INSTR + TB::INSTR;
  constexpr int NF = WM + WN;
  auto issue = [&](int vb, int st) {
#pragma unroll
    for (int j = 0; j < LPB; ++j) issue1(vb, st, j);
  };
  auto fetch = [&](Frags& f, int st, int q) {
#pragma unroll
    for (int i = 0; i < NF; ++i) fetch1(f, st, q, i);
  };
  // the MFMAs of a step; side(i) after the i-th of them, which issues its share
  // of the next step's fragment reads (FT) and direct loads (AT)
  constexpr int NJ = sizeof(E) == 4 ? 4 : 1, NM = NJ * WM * WN;
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

  constexpr int NQ = TA::DEPTH * (int)sizeof(E) / 32;      // steps per K block
  static_assert(NQ % 2 == 0 && (S - 1) * LPB < 64, "pipeline depth");
  Frags fa, fb;
#pragma unroll
  for (int i = 0; i < S; ++i)
    if (i < nblk) issue(vb0 + i, i);
  ahead();
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
    block(it);
  }
}

}  // namespace
}  // namespace hfk
