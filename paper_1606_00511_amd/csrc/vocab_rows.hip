// The row-wise kernels of the softmax head, between its GEMMs.
//
// Rows that do not count (a masked label, an empty teacher list) are left out
// before anything is computed: the counted rows of X are packed one after the
// other, and everything up to the row gradients works on packed rows.  What X
// holds in the others, infinities and NaN included, reaches nothing.
//
// Per packed row, with z the logits over tau and q the targets (q = 1 at the
// label, or the softmax of the teacher's logits over tau within its list):
//   lse   = log sum_v exp z_v, joined from (max, sum) pairs of vocabulary tiles
//   loss  = tau^2 sum_k q_k (log q_k - (z_k - lse))
//   delta = p - q,  p_v = exp(z_v - lse)
// delta is p rounded to the type everywhere but at the targets, where p - q is
// formed in fp32 and rounded once.  With bf16, p comes from exp(z - max) kept
// in fp16 (a rounding of 2^-12 beside delta's 2^-9, down to 2^-29 of the largest
// of the entry) but for few rows.  Losses are summed in fp64.
#include <type_traits>

#include "vocab_internal.h"

namespace hfk {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t f2bf(float f) {
  return __builtin_bit_cast(uint16_t, (__bf16)f);
}
__device__ __forceinline__ float bf2f(uint32_t h) { return __uint_as_float(h << 16); }
__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(bf16_t v) { return bf2f(v); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(bf16_t* p, float v) { *p = (bf16_t)f2bf(v); }

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
  return v;
}
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}
__device__ __forceinline__ double wave_sum_d(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// Target k of row t: its id, or -1 where the place is masked (HF_IGNORE, or a
// teacher logit of -inf); an id outside the vocabulary raises the flag and
// counts as masked.
constexpr int IGNORE = -100;
__device__ __forceinline__ int target(const VRows& r, int t, int k, float* logit) {
  const int id = r.ids[(size_t)t * r.ldi + k];
  if (id == IGNORE) return -1;
  if (id < 0 || id >= r.V) {
    r.st->err = 1;
    return -1;
  }
  if (!r.t) return id;
  const float v = r.t[(size_t)t * r.ldt + k];
  *logit = v;
  return v == -INFINITY ? -1 : id;
}

}  // namespace

// ------------------------------------------------------------ counted rows
// pos[t] = 1 if any of row t's K targets is there, else 0: one wave per row
extern "C" __global__ __launch_bounds__(256) void hf_vocab_have(VRows r) {
  const int t = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (t >= r.T) return;
  bool have = false;
  float v;
  for (int k = lane; k < r.K; k += 64) have |= target(r, t, k, &v) >= 0;
  const bool any = __ballot(have) != 0;
  if (lane == 0) r.pos[t] = any;
}

namespace {
__device__ __forceinline__ void set_state(const VRows& r, int n) {
  const double denom = r.denom > 0.0f ? (double)r.denom : (double)n;
  r.st->n = n;
  r.st->inv = denom > 0.0 ? 1.0 / denom : 0.0;
  r.st->gscale = denom > 0.0 ? (float)((double)r.tau / denom) : 0.0f;
}
// Sum over the threads before this one, and over all, of a workgroup of NW
// waves; sums: NW words of LDS.
template <int NW>
__device__ __forceinline__ int scan_threads(int c, int* sums, int& all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int s = c;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int u = __shfl_up(s, o, 64);
    if (lane >= o) s += u;
  }
  if (lane == 63) sums[wave] = s;
  __syncthreads();
  int base = 0;
  all = 0;
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    if (w < wave) base += sums[w];
    all += sums[w];
  }
  return base + s - c;
}
}  // namespace

// One workgroup of 16 waves: each wave counts a run of rows, 64 at a time, a
// scan over the waves places them.  pos holds hf_vocab_have's answer for
// lists.  (16,384 rows: 16 us; a run of rows per thread, with its scattered
// stores, took 33.)
extern "C" __global__ __launch_bounds__(1024) void hf_vocab_count(VRows r) {
  __shared__ int sums[16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int per = ((r.T + 15) / 16 + 63) & ~63;
  const int t0 = min(wave * per, r.T), t1 = min(t0 + per, r.T);
  constexpr int U = 4;
  // f(row, whether it counts) for the rows of the wave, U x 64 in flight
  auto each = [&](auto f) {
    for (int t = t0; t < t1; t += 64 * U) {
      int v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i = t + 64 * u + lane;
        v[u] = i < t1 ? (r.t ? r.pos[i] : r.ids[(size_t)i * r.ldi]) : 0;
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i = t + 64 * u + lane;
        bool have = v[u] != 0;
        if (!r.t) {
          have = v[u] >= 0 && v[u] < r.V;
          if (i < t1 && !have && v[u] != IGNORE) r.st->err = 1;
        }
        f(i, i < t1, i < t1 && have, v[u]);
      }
    }
  };
  int c = 0, at = 0, n = 0;
  each([&](int, bool, bool have, int) { c += __popcll(__ballot(have)); });
  if (lane == 0) sums[wave] = c;
  __syncthreads();
  for (int w = 0; w < 16; ++w) {
    if (w < wave) at += sums[w];
    n += sums[w];
  }
  each([&](int i, bool in, bool have, int id) {
    const unsigned long long m = __ballot(have);
    const int p = at + __popcll(m & ((1ull << lane) - 1));
    at += __popcll(m);
    if (in) r.pos[i] = have ? p : -1;
    if (have) {
      r.idx[p] = i;
      if (!r.t) r.lab[p] = id;
    } else if (in) {
      r.row_loss[i] = 0.0f;
    }
  });
  if (threadIdx.x == 0) set_state(r, n);
}

// ----------------------------------------------------------------- packing
namespace {
// n elements of src to dst (16-byte aligned, dn elements), zeros past n, by a
// whole workgroup of 256.
template <class E>
__device__ __forceinline__ void copy_row(const E* src, int n, E* dst, int dn, E* dst2) {
  constexpr int EPC = 16 / sizeof(E);
  for (int c = threadIdx.x; c < dn / EPC; c += 256) {
    u32x4 v = u32x4{0u, 0u, 0u, 0u};
    if (EPC * c + EPC <= n) {
      __builtin_memcpy(&v, src + EPC * c, 16);
    } else {
      E w[EPC];
#pragma unroll
      for (int j = 0; j < EPC; ++j) w[j] = EPC * c + j < n ? src[EPC * c + j] : (E)0;
      v = __builtin_bit_cast(u32x4, w);
    }
    *(u32x4*)(dst + EPC * c) = v;
    if (dst2) *(u32x4*)(dst2 + EPC * c) = v;
  }
}

// SELF: up to 256 rows with few targets; every workgroup counts them by
// itself (a launch less), and the first one writes down what later kernels
// need.
constexpr int SELF_ROWS = 256, SELF_TOP = 32;
template <class E, bool SELF>
__device__ __forceinline__ void pack_body(const VRows& r, const E* X, long long ldx,
                                          int in_place, E* xp, int Dp, int dup, E* dX,
                                          long long lddx) {
  const int b = blockIdx.x;
  int n, pos = -1;
  if constexpr (SELF) {
    __shared__ int sums[4], place[SELF_ROWS];
    const int t = threadIdx.x;
    int id = -1;
    float v;
    if (t < r.T)
      for (int k = 0; k < r.K && id < 0; ++k) id = target(r, t, k, &v);
    const bool have = id >= 0;
    const int at = scan_threads<4>(have, sums, n);
    place[t] = have ? at : -1;
    __syncthreads();
    if (b < r.T) pos = place[b];
    if (b == 0) {
      if (t < r.T) {
        if (have) {
          r.idx[at] = t;
          if (!r.t) r.lab[at] = id;
        } else {
          r.row_loss[t] = 0.0f;
        }
      }
      if (t == 0) set_state(r, n);
    }
  } else {
    n = r.st->n;
    if (in_place && n == r.T) return;
    if (b < r.T) pos = r.pos[b];
  }
  if (in_place && n == r.T) return;
  if (b < r.T) {
    if (pos >= 0) {
      copy_row(X + (size_t)b * ldx, r.D, xp + (size_t)pos * Dp, Dp,
               dup ? xp + (size_t)(dup + pos) * Dp : (E*)nullptr);
    } else if (dX) {
      for (int c = threadIdx.x; c < r.D; c += 256) dX[(size_t)b * lddx + c] = (E)0;
    }
    return;
  }
  const int j = n + b - r.T;
  const int end = dup ? dup : (n + VTILE - 1) / VTILE * VTILE;
  if (j < end)
    copy_row((const E*)nullptr, 0, xp + (size_t)j * Dp, Dp,
             dup ? xp + (size_t)(dup + j) * Dp : (E*)nullptr);
}
}  // namespace

#define HF_PACK(SUF, E, SELF)                                                             \
  extern "C" __global__ __launch_bounds__(256) void hf_vocab_pack_##SUF(                  \
      VRows r, const E* X, long long ldx, int in_place, E* xp, int Dp, int dup, E* dX,    \
      long long lddx) {                                                                  \
    pack_body<E, SELF>(r, X, ldx, in_place, xp, Dp, dup, dX, lddx);                       \
  }
HF_PACK(f32, float, false)
HF_PACK(f32_self, float, true)
HF_PACK(bf16, bf16_t, false)
HF_PACK(bf16_self, bf16_t, true)

// Rows of W, padded with zeros to whole K blocks: chunks of 16 bytes, four a
// thread on their way, whatever the rows' width (a workgroup per row took 55 us
// for 50,257 x 1,021 of bf16, 206 MB, and 21 for 58,864 x 214: now 41 and 10).
namespace {
constexpr int COPY_U = 4;
template <class E>
__device__ __forceinline__ void copy_body(const E* W, long long ldw, int R, int D, E* wp,
                                          int Dp) {
  constexpr int EPC = 16 / sizeof(E);
  const int per = Dp / EPC, n = R * per, i0 = blockIdx.x * (256 * COPY_U) + threadIdx.x;
  E v[COPY_U][EPC];
#pragma unroll
  for (int u = 0; u < COPY_U; ++u) {
    const int i = min(i0 + 256 * u, n - 1), row = i / per, c = EPC * (i % per);
    const E* w = W + (size_t)row * ldw + c;
    if (c + EPC <= D) {
      __builtin_memcpy(v[u], w, 16);
    } else {
#pragma unroll
      for (int j = 0; j < EPC; ++j) v[u][j] = c + j < D ? w[j] : (E)0;
    }
  }
#pragma unroll
  for (int u = 0; u < COPY_U; ++u)
    if (i0 + 256 * u < n) *(u32x4*)(wp + (size_t)(i0 + 256 * u) * EPC) = *(const u32x4*)v[u];
}
}  // namespace
extern "C" __global__ __launch_bounds__(256) void hf_vocab_copy_f32(
    const float* W, long long ldw, int R, int D, float* wp, int Dp) {
  copy_body(W, ldw, R, D, wp, Dp);
}
extern "C" __global__ __launch_bounds__(256) void hf_vocab_copy_bf16(
    const bf16_t* W, long long ldw, int R, int D, bf16_t* wp, int Dp) {
  copy_body(W, ldw, R, D, wp, Dp);
}

// ---------------------------------------------------- the targets' logits
// Where the logits are not kept in fp32, those of lists (a label's comes with the
// statistics): the products x_j . W[id] of a packed row, bit for bit as the
// logits' MFMAs sum them.  A logit summed in another order would be off, against
// the sums of the softmax, by as much as is left for the other words where a
// target has nearly all the probability.
//   bf16  the same MFMAs, 32 targets a wave, with the target's row of W as a row
//         of A and its row of X as a column of B, of which the diagonal is used
//   fp32  32 x 32 x 2 MFMAs are a chain of fused multiply-adds, k after k: here
//         one a lane, in the order in which the fragments hold the ks
// Bound by the reads of W's rows (3,686 rows of 64 targets, 2,048 columns of bf16,
// 966 MB: 134 us, 7.2 TB/s from the caches; with 16 bytes of a row a lane straight
// into the fragments, 32 bytes of a line at a time, 170), and where there are few
// by the trips to memory one after the other.
namespace {
// what they are formed of; X: the rows in place where all count, or null
struct VDots {
  const void *X, *xp, *W;
  long long ldx, ldw;
  int Dp;
};
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// 16 bytes of a row from column c on, zeros past its D columns
template <class E>
__device__ __forceinline__ u32x4 row_chunk(const E* row, int c, int D) {
  constexpr int EPC = 16 / sizeof(E);
  u32x4 v = u32x4{0u, 0u, 0u, 0u};
  if (c + EPC <= D) {
    __builtin_memcpy(&v, row + c, 16);
  } else if (c < D) {
    E w[EPC];
#pragma unroll
    for (int i = 0; i < EPC; ++i) w[i] = c + i < D ? row[c + i] : (E)0;
    v = __builtin_bit_cast(u32x4, w);
  }
  return v;
}

// A wave has P pairs: pair p is target p % K of packed row p / K.  RB bytes of
// each pair's row of W at a time come in whole 128-byte lines, through LDS, with
// the next ones on their way; X's rows, which pairs share, straight from the
// caches.  (fp32, 64 pairs and 128 bytes: 300 rows of 32 targets, 768 columns, 17
// us more.)
template <class E>
struct Pairs {
  static constexpr bool F32 = sizeof(E) == 4;
  static constexpr int P = 32, RB = 256;
  static constexpr int EPC = 16 / sizeof(E), CH = RB / 16, N = RB / sizeof(E);
  static constexpr int LOADS = P * CH / 64, STRIDE = RB + 16;   // (STRIDE: LDS banks)
  static constexpr int XL = F32 ? CH : CH / 2;                  // chunks of X a lane needs
};

// f(chunk of X, chunk of W, its number) of the wave's pairs from the first column on;
// lane's pair: lane % P, its chunks: all (fp32, both halves of the wave alike), or
// every second (bf16)
template <class E, class F>
__device__ __forceinline__ void over_pairs(const VRows& r, const VDots& q, int first, int all,
                                           F f) {
  using S = Pairs<E>;
  __shared__ __attribute__((aligned(16))) char lds[4][S::P * S::STRIDE];
  char* const mine = lds[threadIdx.x >> 6];
  const int lane = threadIdx.x & 63, li = lane % S::P, h = lane / S::P;
  const int p = min(first + li, all - 1), j = p / r.K;
  float v;
  // (no target: the first row, its product unused)
  const int id = max(target(r, r.idx[j], p % r.K, &v), 0);
  const E* const x = q.X && r.st->n == r.T ? (const E*)q.X + (size_t)j * q.ldx
                                           : (const E*)q.xp + (size_t)j * q.Dp;
  const E* w[S::LOADS];
#pragma unroll
  for (int i = 0; i < S::LOADS; ++i)
    w[i] = (const E*)q.W + (size_t)__shfl(id, (64 * i + lane) / S::CH, 64) * q.ldw;
  u32x4 a[S::LOADS], b[S::XL];
  auto fetch = [&](int c0) {
#pragma unroll
    for (int i = 0; i < S::LOADS; ++i)
      a[i] = row_chunk(w[i], c0 + S::EPC * ((64 * i + lane) % S::CH), r.D);
#pragma unroll
    for (int g = 0; g < S::XL; ++g)
      b[g] = row_chunk(x, c0 + S::EPC * (S::F32 ? g : 2 * g + h), r.D);
  };
  fetch(0);
  for (int c0 = 0; c0 < r.D; c0 += S::N) {
    u32x4 now[S::XL];
#pragma unroll
    for (int i = 0; i < S::LOADS; ++i)
      *(u32x4*)(mine + (64 * i + lane) / S::CH * S::STRIDE + (64 * i + lane) % S::CH * 16) = a[i];
#pragma unroll
    for (int g = 0; g < S::XL; ++g) now[g] = b[g];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    if (c0 + S::N < r.D) fetch(c0 + S::N);
#pragma unroll
    for (int g = 0; g < S::XL; ++g)
      f(now[g], *(const u32x4*)(mine + li * S::STRIDE + (S::F32 ? g : 2 * g + h) * 16),
        c0 / S::EPC + g);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
}
}  // namespace

extern "C" __global__ __launch_bounds__(256) void hf_vocab_tlogit_bf16(VRows r, VDots q,
                                                                       float zscale, float* zt) {
  const int lane = threadIdx.x & 63, li = lane & 31, h = lane >> 5;
  const int first = (blockIdx.x * 4 + (threadIdx.x >> 6)) * 32, all = r.st->n * r.K;
  if (first >= all) return;
  f32x16 acc;
#pragma unroll
  for (int i = 0; i < 16; ++i) acc[i] = 0.0f;
  over_pairs<bf16_t>(r, q, first, all, [&](u32x4 x, u32x4 w, int) {
    acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, w),
                                                  __builtin_bit_cast(bf16x8, x), acc, 0, 0, 0);
  });
  // lane (li, h), register i holds row 8 (i / 4) + 4 h + i % 4 of column li
  float v = 0.0f;
#pragma unroll
  for (int i = 0; i < 16; ++i)
    if (4 * (li >> 3) + (li & 3) == i) v = acc[i];
  if (((li >> 2) & 1) == h && first + li < all) zt[first + li] = v * zscale;
}

extern "C" __global__ __launch_bounds__(256) void hf_vocab_tlogit_f32(VRows r, VDots q, int parts,
                                                                      float zscale, float* zt) {
  const int lane = threadIdx.x & 63;
  const int first = (blockIdx.x * 4 + (threadIdx.x >> 6)) * 32, all = r.st->n * r.K;
  if (first >= all) return;
  float s = 0.0f, before = 0.0f;
  f32x4 x0, w0;            // of the chunk before
  over_pairs<float>(r, q, first, all, [&](u32x4 x, u32x4 w, int g) {
    const f32x4 xf = __builtin_bit_cast(f32x4, x), wf = __builtin_bit_cast(f32x4, w);
    // a lane of half 0 of the MFMAs has columns 8 q .. 8 q + 3 of step q, one of
    // half 1 the next four; MFMA i takes the i-th of both
    if (g & 1) {
#pragma unroll
      for (int i = 0; i < 4; ++i) s = __builtin_fmaf(wf[i], xf[i], __builtin_fmaf(w0[i], x0[i], s));
    }
    if (parts && (g + 1) % (SUM_COLS / 4) == 0) {
      before += s;
      s = 0.0f;
    }
    x0 = xf;
    w0 = wf;
  });
  if (parts) s = before + s;
  if (lane < 32 && first + lane < all) zt[first + lane] = s * zscale;
}

// ------------------------------------------------------------- rows' losses
namespace {
struct RowTargets {          // lane l: targets l and l + 64
  float lse, loss;
  int id[2];                 // -1: none, or a repeat
  float dt[2];               // delta at the target
};
// One packed row j < n by one wave.  The targets' logits: in zt, or (null) in z.
__device__ __forceinline__ RowTargets row_targets(const VRows& r, int j,
                                                  const float2* __restrict__ stat, int ldstat,
                                                  int tiles, const float* __restrict__ z,
                                                  long long ldz,
                                                  const float* __restrict__ zt) {
  const int lane = threadIdx.x & 63, t = r.idx[j];
  RowTargets o;
  const float2* st = stat + (size_t)j * ldstat;
  // 8 entries a lane at a time; (m, s) of those before are scaled to the new
  // maximum (0 instead of -inf: exp(-inf - 0) = 0)
  constexpr int U = 8;
  float m = -INFINITY, s = 0.0f;
  for (int i0 = lane; i0 < tiles; i0 += 64 * U) {
    float2 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      v[u] = i0 + 64 * u < tiles ? st[i0 + 64 * u] : float2{-INFINITY, 0.0f};
    float top = m;
#pragma unroll
    for (int u = 0; u < U; ++u) top = fmaxf(top, v[u].x);
    const float at = top == -INFINITY ? 0.0f : top;
    s *= expf(m - at);
#pragma unroll
    for (int u = 0; u < U; ++u) s += v[u].y * expf(v[u].x - at);
    m = top;
  }
  const float mx = wave_max(m), at = mx == -INFINITY ? 0.0f : mx;
  const float ls = logf(wave_sum(s * expf(m - at)));
  o.lse = at + ls;

  int id[2] = {-1, -1};
  float tl[2] = {0.0f, 0.0f}, q[2] = {0.0f, 0.0f}, lz[2] = {0.0f, 0.0f};
#pragma unroll
  for (int i = 0; i < 2; ++i)
    if (lane + 64 * i < r.K) {
      const int k = lane + 64 * i;
      id[i] = target(r, t, k, &tl[i]);
      if (id[i] >= 0) {
        const float x = zt ? zt[(size_t)j * r.K + k] : z[(size_t)j * ldz + id[i]];
        // log p, of the difference to the largest, which for a target with nearly
        // all the probability is 0 where lse is rounded to its own size; above 0
        // only by rounding (the comparison keeps a NaN)
        const float lp = (x - at) - ls;
        lz[i] = lp > 0.0f ? 0.0f : lp;
      }
    }
  float loss = 0.0f;
  // an id that comes twice: its first place has the sum of its q
  float qs[2] = {id[0] >= 0 ? 1.0f : 0.0f, 0.0f};
  int first[2] = {1, 1};
  if (!r.t) {
    loss = -lz[0];
  } else {
    // differences before the division: a logit of the type's lowest value
    // over a small tau is no infinity then
    const float top = wave_max(fmaxf(id[0] >= 0 ? tl[0] : -INFINITY,
                                     id[1] >= 0 ? tl[1] : -INFINITY));
    float e[2], u[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      u[i] = (tl[i] - top) / r.tau;
      e[i] = id[i] >= 0 ? expf(u[i]) : 0.0f;
    }
    const float total = wave_sum(e[0] + e[1]);
    const float lt = logf(total);
    int same[2] = {0, 0};
    qs[0] = 0.0f;
#pragma unroll
    for (int i2 = 0; i2 < 2; ++i2) {
      q[i2] = e[i2] / total;
      for (int l = 0; l < 64 && l + 64 * i2 < r.K; ++l) {
        const int oid = __shfl(id[i2], l, 64);
        const float oq = __shfl(q[i2], l, 64);
#pragma unroll
        for (int i = 0; i < 2; ++i)
          if (oid == id[i]) {
            qs[i] += oq;
            ++same[i];
            if (l + 64 * i2 < lane + 64 * i) first[i] = 0;
          }
      }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (id[i] >= 0 && first[i] && qs[i] != 0.0f)
        loss += qs[i] * ((same[i] > 1 ? logf(qs[i]) : u[i] - lt) - lz[i]);
  }
  loss = wave_sum(loss) * (r.tau * r.tau);
  o.loss = loss < 0.0f ? 0.0f : loss;    // no divergence is; rounding can be
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    o.id[i] = first[i] ? id[i] : -1;
    o.dt[i] = expf(lz[i]) - qs[i];
  }
  return o;
}
}  // namespace

// The loss from the rows' losses, by one workgroup of 256 threads.
namespace {
__device__ __forceinline__ void loss_sum(const float* row_loss, int T, const VocabState* st,
                                         float* loss) {
  __shared__ double ws[4];
  double s = 0.0;
  for (int t = threadIdx.x; t < T; t += 8 * 256) {
    float v[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] = t + 256 * u < T ? row_loss[t + 256 * u] : 0.0f;
#pragma unroll
    for (int u = 0; u < 8; ++u) s += (double)v[u];
  }
  s = wave_sum_d(s);
  if ((threadIdx.x & 63) == 0) ws[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) *loss = (float)(((ws[0] + ws[1]) + (ws[2] + ws[3])) * st->inv);
}
}  // namespace
// One wave per packed row.  With `loss` (few rows, one workgroup) the rows' losses
// are summed as well.
extern "C" __global__ __launch_bounds__(256) void hf_vocab_row_loss(
    VRows r, const float2* stat, int ldstat, int tiles, const float* z, long long ldz,
    VTarget tg, float* lse, float* loss) {
  const int lane = threadIdx.x & 63, waves = blockDim.x >> 6;
  for (int j = blockIdx.x * waves + (threadIdx.x >> 6); j < r.st->n; j += gridDim.x * waves) {
    const RowTargets o = row_targets(r, j, stat, ldstat, tiles, z, ldz, z ? nullptr : tg.zt);
    if (lane == 0) {
      lse[j] = o.lse;
      r.row_loss[r.idx[j]] = o.loss;
    }
    if (!tg.dt) continue;
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (lane + 64 * i < r.K) {
        tg.id[(size_t)j * r.K + lane + 64 * i] = o.id[i];
        tg.dt[(size_t)j * r.K + lane + 64 * i] = o.dt[i];
      }
  }
  if (loss) {
    __syncthreads();
    loss_sum(r.row_loss, r.T, r.st, loss);
  }
}

extern "C" __global__ __launch_bounds__(256) void hf_vocab_loss_sum(
    const float* __restrict__ row_loss, int T, const VocabState* st, float* loss) {
  loss_sum(row_loss, T, st, loss);
}

// ------------------------------------------------------------------- delta
// A workgroup has 2,048 of the Vc columns from v0 of one packed row; z and d
// hold these columns from 0.
// SELF (few rows): it forms the row's statistics and targets by itself (a
// launch less), the first columns' workgroup writes the row's loss; otherwise
// they come from hf_vocab_row_loss, and the last workgroup sums the loss.
namespace {
constexpr int DCOLS = 2048;
struct VDelta {
  const float* z;
  long long ldz;
  const float2* stat;
  int ldstat, tiles;
  const float* lse;
  VTarget tg;
  int chunks, v0, Vc, Vp, dup;
  long long ldd;
  float* loss;
  int sg;                      // columns of a statistics entry
};
// FROM16: d holds EXP_SCALE exp(z - max) in fp16 and becomes delta in place.
template <class E, bool SELF, bool FROM16>
__device__ __forceinline__ void delta_body(const VRows& r, const VDelta& a, E* d) {
  if (!SELF && a.loss && blockIdx.x == gridDim.x - 1) {
    loss_sum(r.row_loss, r.T, r.st, a.loss);
    return;
  }
  __shared__ float lse_s, dt_s[SELF ? 128 : 1];
  __shared__ int id_s[SELF ? 128 : 1];
  const int j = blockIdx.x / a.chunks, c0 = (blockIdx.x % a.chunks) * DCOLS;
  const int n = r.st->n;
  if (j >= n && j >= (a.dup ? a.dup : (n + VPAD - 1) / VPAD * VPAD)) return;
  const bool real = j < n;
  if constexpr (SELF) {
    if (real && threadIdx.x < 64) {
      const int lane = threadIdx.x;
      const RowTargets o = row_targets(r, j, a.stat, a.ldstat, a.tiles, a.z, a.ldz, nullptr);
      if (lane == 0) {
        lse_s = o.lse;
        if (c0 == 0) r.row_loss[r.idx[j]] = o.loss;
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        id_s[lane + 64 * i] = o.id[i];
        dt_s[lane + 64 * i] = o.dt[i];
      }
    }
    __syncthreads();
  }
  const float l = !real ? 0.0f : SELF ? lse_s : a.lse[j];
  E* hi = d + (size_t)j * a.ldd;
  E* lo = a.dup ? d + (size_t)(a.dup + j) * a.ldd : nullptr;
  const float* zr = a.z + (size_t)j * a.ldz;
  if constexpr (FROM16) {
    // 8 columns a thread, of one statistics entry
    typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
    const int c = c0 + 8 * (int)threadIdx.x;
    if (c < a.Vp) {
      u32x4 w = u32x4{0u, 0u, 0u, 0u};
      if (real && c < a.Vc) {
        const float f = expf(a.stat[(size_t)j * a.ldstat + (a.v0 + c) / a.sg].x - l) *
                        (1.0f / EXP_SCALE);
        const f16x8 x = *(const f16x8*)(hi + c);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          w[e] = f2bf((float)x[2 * e] * f) | f2bf((float)x[2 * e + 1] * f) << 16;
      }
      *(u32x4*)(hi + c) = w;
    }
  }
  // 4 columns a thread and step
#pragma unroll
  for (int i = 0; !FROM16 && i < DCOLS / 1024; ++i) {
    const int c = c0 + 4 * (int)threadIdx.x + 1024 * i;
    if (c >= a.Vp) break;
    float v[4];
    f32x4 zz = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    if (real) zz = *(const f32x4*)(zr + c);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = real && c + e < a.Vc ? expf(zz[e] - l) : 0.0f;
    if constexpr (sizeof(E) == 4) {
      *(f32x4*)(hi + c) = f32x4{v[0], v[1], v[2], v[3]};
    } else {
      uint32_t b[4], s[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        b[e] = f2bf(v[e]);
        s[e] = f2bf(v[e] - bf2f(b[e]));
      }
      *(u32x2*)(hi + c) = u32x2{b[0] | b[1] << 16, b[2] | b[3] << 16};
      if (lo) *(u32x2*)(lo + c) = u32x2{s[0] | s[1] << 16, s[2] | s[3] << 16};
    }
  }
  if (!real) return;
  // the targets among these columns, over what was just written
  __syncthreads();
  for (int k = threadIdx.x; k < r.K; k += 256) {
    const int id = SELF ? id_s[k] : a.tg.id[(size_t)j * r.K + k];
    if (id < 0 || id < a.v0 + c0 || id >= a.v0 + min(c0 + DCOLS, a.Vc)) continue;
    const float v = SELF ? dt_s[k] : a.tg.dt[(size_t)j * r.K + k];
    put(hi + (id - a.v0), v);
    if constexpr (sizeof(E) == 2)
      if (lo) put(lo + (id - a.v0), v - bf2f(f2bf(v)));
  }
}
}  // namespace
#define HF_DELTA(SUF, E, SELF, FROM16)                                      \
  extern "C" __global__ __launch_bounds__(256) void hf_vocab_delta_##SUF(   \
      VRows r, VDelta a, E* d) {                                            \
    delta_body<E, SELF, FROM16>(r, a, d);                                   \
  }
HF_DELTA(f32, float, false, false)
HF_DELTA(bf16, bf16_t, false, true)
HF_DELTA(bf16_self, bf16_t, true, false)

namespace {
template <class E>
__device__ __forceinline__ void fix_body(const VRows& r, const VTarget& tg, int v0, int Vc, E* d,
                                         long long ldd) {
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
  if (i >= (long long)r.st->n * r.K) return;
  const int id = tg.id[i];
  if (id >= v0 && id < v0 + Vc) put(d + (size_t)(i / r.K) * ldd + (id - v0), tg.dt[i]);
}
}  // namespace
extern "C" __global__ __launch_bounds__(256) void hf_vocab_fix_f32(VRows r, VTarget tg, int v0,
                                                                   int Vc, float* d,
                                                                   long long ldd) {
  fix_body<float>(r, tg, v0, Vc, d, ldd);
}
extern "C" __global__ __launch_bounds__(256) void hf_vocab_fix_bf16(VRows r, VTarget tg, int v0,
                                                                    int Vc, bf16_t* d,
                                                                    long long ldd) {
  fix_body<bf16_t>(r, tg, v0, Vc, d, ldd);
}

// ------------------------------------------------------------------ finish
// 4 columns of a row per group of G threads, each of which adds every G-th
// partial (the splits, then the dup copy's) in order; then the G sums in
// order.  With one partial per thread in turn, 128 partials took 36 us of
// latency; G = 8 takes 5.
namespace {
struct VParts {
  const float* part;
  long long ldp;
  int splits, smax, n, rn, dyn;   // of the product: n rows in tiles of rn
  int direct;                     // one split: nothing is left to do
};
template <class E, int G>
__device__ __forceinline__ void finish_body(const VocabState* st, const VParts& p, int dup,
                                            int rows, int counted, int D, const int* idx, E* out,
                                            long long ldo, int accumulate,
                                            const float* row_loss, int T, float* loss) {
  if (loss && blockIdx.x == gridDim.x - 1) {
    loss_sum(row_loss, T, st, loss);
    return;
  }
  constexpr int QB = 256 / G;           // column groups per workgroup
  const int groups = gridDim.x - (loss ? 1 : 0);
  __shared__ f32x4 sums[G > 1 ? 256 : 1];
  const int q = (D + 3) / 4, grp = threadIdx.x / QB;
  if (counted) rows = min(st->n, rows);
  const int gy = (p.n + p.rn - 1) / p.rn;
  const int gya = p.dyn == 1 ? (st->n + p.rn - 1) / p.rn : gy;
  const int splits = splits_of(p.splits, p.smax, gy, gya);
  if (p.direct && splits == 1) return;
  const size_t ss = (size_t)gya * p.rn * p.ldp;
  const int parts = dup ? 2 * splits : splits;
  const float g = st->gscale;
  // (once, except where the direct store was likelier, and for very large outputs)
  for (long long i0 = (long long)blockIdx.x * QB; i0 < (long long)rows * q;
       i0 += (long long)groups * QB) {
    const long long i = i0 + threadIdx.x % QB;
    const int j = (int)(i / q), c = 4 * (int)(i % q);
    const bool in = j < rows;
    f32x4 s = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    if (in) {
      constexpr int U = G > 1 ? 8 : 4;
      for (int z0 = grp; z0 < parts; z0 += U * G) {
        f32x4 v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int z = min(z0 + u * G, parts - 1), zz = z < splits ? z : z - splits;
          const size_t row = z < splits ? j : dup + j;
          v[u] = *(const f32x4*)(p.part + zz * ss + row * p.ldp + c);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (z0 + u * G < parts) s += v[u];
      }
    }
    if constexpr (G > 1) {
      __syncthreads();
      sums[threadIdx.x] = s;
      __syncthreads();
      if (!grp)
        for (int k = 1; k < G; ++k) s += sums[k * QB + threadIdx.x];
    }
    if (!in || grp) continue;
    E* o = out + (size_t)(idx ? idx[j] : j) * ldo + c;
    E w[4] = {};
    if (accumulate) {
      if (c + 4 <= D) __builtin_memcpy(w, o, sizeof w);
      else
        for (int e = 0; e < 3; ++e)
          if (c + e < D) w[e] = o[e];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) put(w + e, s[e] * g + (accumulate ? to_f(w[e]) : 0.0f));
    if (c + 4 <= D) __builtin_memcpy(o, w, sizeof w);
    else
      for (int e = 0; e < 3; ++e)
        if (c + e < D) o[e] = w[e];
  }
}
}  // namespace
#define HF_FINISH(SUF, E, G)                                                               \
  extern "C" __global__ __launch_bounds__(256) void hf_vocab_finish_##SUF(                 \
      const VocabState* st, VParts p, int dup, int rows, int counted, int D,               \
      const int* idx, E* out, long long ldo, int accumulate, const float* row_loss, int T, \
      float* loss) {                                                                       \
    finish_body<E, G>(st, p, dup, rows, counted, D, idx, out, ldo, accumulate, row_loss,   \
                      T, loss);                                                            \
  }
HF_FINISH(f32, float, 1)
HF_FINISH(f32_g8, float, 8)
HF_FINISH(bf16, bf16_t, 1)
HF_FINISH(bf16_g8, bf16_t, 8)

// ------------------------------------------------------------- launchers
#define HF_LAUNCH(NAME, K, GRID, BLOCK, ...)                                       \
  do {                                                                             \
    prof_begin(L, NAME);                                                           \
    hipExtLaunchKernelGGL(K, dim3((unsigned)(GRID)), dim3(BLOCK), 0, L.stream,     \
                          prof_a(L), prof_b(L), 0, __VA_ARGS__);                   \
    prof_end(L, NAME, 0.0, 0.0);                                                   \
  } while (0)

namespace {
constexpr int SUM_ROWS = 16;      // rows whose losses one workgroup forms and sums
}  // namespace

bool vocab_count(const Launch& L, const VRows& r) {
  if (r.T > 0 && r.T <= SELF_ROWS && r.K <= SELF_TOP) return false;
  if (r.t && r.T > 0)
    HF_LAUNCH("hf_vocab_have", hf_vocab_have, (r.T + 3) / 4, 256, r);
  HF_LAUNCH("hf_vocab_count", hf_vocab_count, 1, 1024, r);
  return true;
}

void vocab_pack_rows(const Launch& L, int type, const VRows& r, bool counted, const void* X,
                     long long ldx, bool in_place, void* xp, int Dp, int dup, void* dX,
                     long long lddx) {
  const int grid = r.T + (dup ? dup : VTILE), place = in_place;
  if (type == VT_F32)
    HF_LAUNCH("hf_vocab_pack", (counted ? hf_vocab_pack_f32 : hf_vocab_pack_f32_self), grid,
              256, r, (const float*)X, ldx, place, (float*)xp, Dp, dup,
              (float*)dX, lddx);
  else
    HF_LAUNCH("hf_vocab_pack", (counted ? hf_vocab_pack_bf16 : hf_vocab_pack_bf16_self), grid,
              256, r, (const bf16_t*)X, ldx, place, (bf16_t*)xp, Dp, dup,
              (bf16_t*)dX, lddx);
}

void vocab_pack_matrix(const Launch& L, int type, const void* W, long long ldw, int R, int D,
                       void* wp, int Dp) {
  const int es = type == VT_F32 ? 4 : 2, chunks = R * (Dp * es / 16);   // of 256 MiB at most
  const int grid = (chunks + 256 * COPY_U - 1) / (256 * COPY_U);
  if (type == VT_F32)
    HF_LAUNCH("hf_vocab_copy", hf_vocab_copy_f32, grid, 256, (const float*)W, ldw, R, D,
              (float*)wp, Dp);
  else
    HF_LAUNCH("hf_vocab_copy", hf_vocab_copy_bf16, grid, 256, (const bf16_t*)W, ldw, R, D,
              (bf16_t*)wp, Dp);
}

bool vocab_row_loss(const Launch& L, int type, const VRows& r, bool parts, const float2* stat,
                    int ldstat, int tiles, const float* z, long long ldz, const VTarget& t, float* lse,
                    const void* X, long long ldx, const void* xp, int Dp, const void* W,
                    long long ldw, float* loss) {
  if (r.T < 1) return false;
  const VDots q = {X, xp, W, ldx, ldw, Dp};
  if (!z && r.t) {
    const long long pairs = (long long)r.T * r.K;
    const float zscale = 1.0f / r.tau;        // as the logits'
    if (type == VT_F32)
      HF_LAUNCH("hf_vocab_tlogit", hf_vocab_tlogit_f32, (pairs + 127) / 128, 256, r, q,
                (int)parts, zscale, t.zt);
    else
      HF_LAUNCH("hf_vocab_tlogit", hf_vocab_tlogit_bf16, (pairs + 127) / 128, 256, r, q, zscale,
                t.zt);
  }
  const bool sum = loss && r.T <= SUM_ROWS;
  HF_LAUNCH("hf_vocab_row_loss", hf_vocab_row_loss, sum ? 1 : (r.T + 3) / 4, 256, r, stat, ldstat,
            tiles, z, ldz, t, lse, sum ? loss : nullptr);
  return sum;
}

void vocab_loss_sum(const Launch& L, const VRows& r, float* loss) {
  HF_LAUNCH("hf_vocab_loss_sum", hf_vocab_loss_sum, 1, 256, r.row_loss, r.T, r.st, loss);
}

void vocab_delta(const Launch& L, int type, const VRows& r, const float* z, long long ldz,
                 const float2* stat, int tiles, int sg, const float* lse, const VTarget& t, int v0,
                 int Vc, int rows, bool self, void* d, long long ldd, int dup, float* loss) {
  VDelta a = {};
  a.z = z;
  a.ldz = ldz;
  a.stat = stat;
  a.ldstat = a.tiles = tiles;
  a.lse = lse;
  a.tg = t;
  a.Vp = (Vc + VPAD - 1) / VPAD * VPAD;
  a.chunks = (a.Vp + DCOLS - 1) / DCOLS;
  a.v0 = v0;
  a.Vc = Vc;
  a.dup = dup;
  a.ldd = ldd;
  a.loss = loss;
  a.sg = sg;
  const long long grid = (long long)rows * a.chunks + (loss && !self ? 1 : 0);
  if (type == VT_F32)
    HF_LAUNCH("hf_vocab_delta", hf_vocab_delta_f32, grid, 256, r, a, (float*)d);
  else
    HF_LAUNCH("hf_vocab_delta", (self ? hf_vocab_delta_bf16_self : hf_vocab_delta_bf16), grid,
              256, r, a, (bf16_t*)d);
}

void vocab_fix(const Launch& L, int type, const VRows& r, const VTarget& t, int v0, int Vc,
               void* d, long long ldd) {
  const long long grid = ((long long)r.T * r.K + 255) / 256;
  if (type == VT_F32)
    HF_LAUNCH("hf_vocab_fix", hf_vocab_fix_f32, grid, 256, r, t, v0, Vc, (float*)d, ldd);
  else
    HF_LAUNCH("hf_vocab_fix", hf_vocab_fix_bf16, grid, 256, r, t, v0, Vc, (bf16_t*)d, ldd);
}

void vocab_finish(const Launch& L, int type, const VGemm& g, const VEpi& e, int dup, int rows,
                  int counted, int D, const int* idx, void* out, long long ldo, int accumulate,
                  const VRows* r, float* loss) {
  const VParts p = {e.part, e.ldp, g.splits, g.smax, g.N, tile_n(g.tile), g.dyn, e.out != nullptr};
  const bool g8 = (dup ? 2 : 1) * g.splits >= 16;
  long long grid = ((long long)rows * ((D + 3) / 4) * (g8 ? 8 : 1) + 255) / 256;
  // a launch has fewer than 2^32 work-items (262,144 rows of 65,536 columns would
  // have as many); and most often nothing is left to do after a direct store:
  // 16,384 workgroups that end at once take 12 us, 2,048 take 4.5
  grid = std::min<long long>(grid, p.direct && g.splits == 1 ? 2048 : 1 << 20) + (loss ? 1 : 0);
  if (grid < 1) return;
  const float* rl = loss ? r->row_loss : nullptr;
  const int T = loss ? r->T : 0;
  if (type == VT_F32)
    HF_LAUNCH("hf_vocab_finish", (g8 ? hf_vocab_finish_f32_g8 : hf_vocab_finish_f32), grid, 256,
              g.st, p, dup, rows, counted, D, idx, (float*)out, ldo, accumulate, rl, T, loss);
  else
    HF_LAUNCH("hf_vocab_finish", (g8 ? hf_vocab_finish_bf16_g8 : hf_vocab_finish_bf16), grid,
              256, g.st, p, dup, rows, counted, D, idx, (bf16_t*)out, ldo, accumulate, rl, T,
              loss);
}

}  // namespace hfk
