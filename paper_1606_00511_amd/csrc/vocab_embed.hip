// Token embedding and its gradient.
//   forward   out_t = scale E[tok_t], zeros where the token is masked
//   gradient  dE_v = scale sum_{t: tok_t = v} dout_t, in token order, fp32
// Both are bound by memory: each row is read and written once.
//
// The gradient sorts the rows by token (stable, two radix passes), so that the
// rows of one token are consecutive, and cuts the sorted places into runs of
// RUN.  A wave sums a run, strip of columns by strip, and writes the tokens
// that lie within it; what reaches over a run's ends goes to partial sums,
// which a last kernel joins in order.  So the work per wave does not depend on
// how often a token comes, and no sum uses atomics: the same bits every time.
// The sort occupies few compute units and waits for memory most of the time:
// the other workgroups of its launches fill dE with zeros meanwhile (rows of
// tokens that do come are written again: fewer than there are rows of dout).
#include <algorithm>

#include "vocab_internal.h"

namespace hfk {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 __attribute__((aligned(2))) loose;      // of any alignment

__device__ __forceinline__ uint32_t f2bf(float f) {
  return __builtin_bit_cast(uint16_t, (__bf16)f);
}
__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(bf16_t v) { return __uint_as_float((uint32_t)v << 16); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(bf16_t* p, float v) { *p = (bf16_t)f2bf(v); }

constexpr int IGNORE = -100;

// A wave has EPC columns of a row per lane and strip: 16 consecutive bytes,
// whatever their alignment (VEC), else single elements 64 apart.  The lane with
// a row's end takes the last 16 bytes; it and the lane before it then compute
// the same, and write the same, in one instruction.  So VEC is for rows whose
// end shares a strip with a whole chunk (30,000 x 1,021 of bf16: embedding
// 32 -> 18 us, gradient 66 -> 58).  STREAM: past the caches.
template <class E, bool VEC>
struct Strip {
  static constexpr int EPC = 16 / (int)sizeof(E);
  static constexpr int COLS = 64 * EPC;
  __device__ static __forceinline__ int col(int strip, int lane, int e) {
    return strip * COLS + (VEC ? lane * EPC + e : e * 64 + lane);
  }
  // (VEC) the lane's first column
  __device__ static __forceinline__ int first(int strip, int lane, int D) {
    return min(col(strip, lane, 0), D - EPC);
  }
  struct Raw {               // as loaded: 4 registers for a lane's columns
    E v[EPC];
  };
  template <bool STREAM>
  __device__ static __forceinline__ Raw raw(const E* row, int strip, int lane, int D) {
    Raw w = {};
    if constexpr (VEC) {
      if (col(strip, lane, 0) < D) {
        const loose* const p = (const loose*)(row + first(strip, lane, D));
        w = __builtin_bit_cast(Raw, STREAM ? __builtin_nontemporal_load(p) : *p);
      }
    } else {
#pragma unroll
      for (int e = 0; e < EPC; ++e) {
        const int c = col(strip, lane, e);
        if (c < D) w.v[e] = row[c];
      }
    }
    return w;
  }
  __device__ static __forceinline__ void load(const E* row, int strip, int lane, int D,
                                              float (&v)[EPC]) {
    const Raw w = raw<false>(row, strip, lane, D);
#pragma unroll
    for (int e = 0; e < EPC; ++e) v[e] = to_f(w.v[e]);
  }
  template <bool STREAM>
  __device__ static __forceinline__ void store(E* row, int strip, int lane, int D,
                                               const float (&v)[EPC]) {
    if constexpr (VEC) {
      E w[EPC];
#pragma unroll
      for (int e = 0; e < EPC; ++e) put(w + e, v[e]);
      if (col(strip, lane, 0) < D) {
        loose* const p = (loose*)(row + first(strip, lane, D));
        const u32x4 x = __builtin_bit_cast(u32x4, w);
        if (STREAM) __builtin_nontemporal_store(x, p);
        else *p = x;
      }
    } else {
#pragma unroll
      for (int e = 0; e < EPC; ++e) {
        const int c = col(strip, lane, e);
        if (c < D) put(row + c, v[e]);
      }
    }
  }
};

// One strip of one row per wave.
template <class E, bool VEC, bool STREAM>
__device__ __forceinline__ void embed_body(const E* table, long long lde, int V, int D,
                                           const int32_t* tok, int T, int strips, float scale,
                                           E* out, long long ldo, VocabState* st) {
  using S = Strip<E, VEC>;
  const int lane = threadIdx.x & 63;
  const long long u = ((long long)blockIdx.y * gridDim.x + blockIdx.x) * 4 + (threadIdx.x >> 6);
  const int t = (int)(u / strips), strip = (int)(u % strips);
  if (t >= T) return;
  const int id = __builtin_amdgcn_readfirstlane(tok[t]);
  float v[S::EPC];
  if (id >= 0 && id < V) {
    S::load(table + (size_t)id * lde, strip, lane, D, v);
  } else {
    if (id != IGNORE && lane == 0) st->err = 1;
#pragma unroll
    for (int e = 0; e < S::EPC; ++e) v[e] = 0.0f;
  }
#pragma unroll
  for (int e = 0; e < S::EPC; ++e) v[e] *= scale;
  S::template store<STREAM>(out + (size_t)t * ldo, strip, lane, D, v);
}

}  // namespace

#define HF_EMBED(SUF, E, VEC, STREAM)                                                    \
  extern "C" __global__ __launch_bounds__(256) void hf_vocab_embed_##SUF(                \
      const E* table, long long lde, int V, int D, const int32_t* tok, int T, int strips, \
      float scale, E* out, long long ldo, VocabState* st) {                              \
    embed_body<E, VEC, STREAM>(table, lde, V, D, tok, T, strips, scale, out, ldo, st);   \
  }
HF_EMBED(f32, float, false, false)
HF_EMBED(f32_v, float, true, false)
HF_EMBED(f32_s, float, true, true)
HF_EMBED(bf16, bf16_t, false, false)
HF_EMBED(bf16_v, bf16_t, true, false)
HF_EMBED(bf16_s, bf16_t, true, true)

// -------------------------------------------------------------------- sort
// Least-significant digit first, two digits of `bits` bits.  The key is the
// token; masked ones take V, past every row.  A workgroup of 16 waves has
// 1,024 places; hist[b * digits + d] counts digit d in workgroup b's places.
namespace {
constexpr int CHUNK = 1024;
constexpr int MAXDIG = 4096;

__device__ __forceinline__ int key_of(const int32_t* tok, int t, int V, VocabState* st) {
  const int id = tok[t];
  if (id >= 0 && id < V) return id;
  if (id != IGNORE) st->err = 1;
  return V;
}

// A share of the rows of dE set to zero by the workgroups past the sort's.
struct Fill {
  char* p;             // null: nothing to fill
  long long ld;        // bytes between rows
  int bytes;           // of a row
  int v0, v1;          // rows
};
__device__ __forceinline__ void fill_rows(const Fill& f, int block, int blocks) {
  const int lane = threadIdx.x & 63;
  for (int v = f.v0 + block * (CHUNK / 64) + (threadIdx.x >> 6); v < f.v1;
       v += blocks * (CHUNK / 64)) {
    char* row = f.p + (size_t)v * f.ld;
    const u32x4 zero = u32x4{0u, 0u, 0u, 0u};
    for (int i = 16 * lane; i < f.bytes; i += 1024) {
      if (i + 16 <= f.bytes) *(loose*)(row + i) = zero;
      else
        for (int j = i; j < f.bytes; j += 2) *(uint16_t*)(row + j) = 0;
    }
  }
}

// Exclusive scan of a[0 .. n), n <= MAXDIG, by 1,024 threads.
__device__ __forceinline__ void scan_digits(unsigned* a, int n, unsigned* tmp) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int per = (n + 1023) / 1024;
  unsigned c = 0;
  for (int i = 0; i < per; ++i)
    if (tid * per + i < n) c += a[tid * per + i];
  unsigned s = c;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const unsigned u = __shfl_up(s, o, 64);
    if (lane >= o) s += u;
  }
  if (lane == 63) tmp[wave] = s;
  __syncthreads();
  unsigned base = 0;
  for (int w = 0; w < wave; ++w) base += tmp[w];
  unsigned at = base + s - c;
  __syncthreads();
  for (int i = 0; i < per; ++i)
    if (tid * per + i < n) {
      const unsigned x = a[tid * per + i];
      a[tid * per + i] = at;
      at += x;
    }
  __syncthreads();
}

// Lanes whose first `bits` bits of v agree with this lane's, of those in m.
__device__ __forceinline__ unsigned long long alike(unsigned long long m, unsigned v, int bits) {
  for (int b = 0; b < bits; ++b) {
    const unsigned long long one = __ballot((v >> b) & 1);
    m &= ((v >> b) & 1) ? one : ~one;
  }
  return m;
}

// The place of each thread's element among the elements of its digit: `base`
// holds where each digit's next element goes.  The waves take their turns in
// order, so that equal digits keep their order.
__device__ __forceinline__ unsigned place(unsigned* base, int d, bool valid, int bits) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const unsigned long long same = alike(__ballot(valid), (unsigned)d, bits);
  const unsigned below = __popcll(same & ((1ull << lane) - 1));
  unsigned at = 0;
  for (int w = 0; w < CHUNK / 64; ++w) {
    if (w == wave && valid) {
      at = base[d] + below;
      // every lane of the wave has read before its first of a digit advances it
      __builtin_amdgcn_wave_barrier();
      if (below == 0) base[d] += __popcll(same);
    }
    __syncthreads();
  }
  return at;
}
}  // namespace

// histogram of the low digit; zeros in the high digit's
extern "C" __global__ __launch_bounds__(CHUNK) void hf_vocab_sort_hist(
    const int32_t* tok, int T, int V, int bits, unsigned* hist, unsigned* hist2, int blocks,
    Fill fill, VocabState* st) {
  if ((int)blockIdx.x >= blocks) {
    fill_rows(fill, blockIdx.x - blocks, gridDim.x - blocks);
    return;
  }
  __shared__ unsigned h[MAXDIG];
  const int digs = 1 << bits, t = blockIdx.x * CHUNK + threadIdx.x;
  for (int d = threadIdx.x; d < digs; d += CHUNK) h[d] = 0;
  __syncthreads();
  if (t < T) atomicAdd(&h[key_of(tok, t, V, st) & (digs - 1)], 1u);
  __syncthreads();
  for (int d = threadIdx.x; d < digs; d += CHUNK) {
    hist[(size_t)blockIdx.x * digs + d] = h[d];
    hist2[(size_t)blockIdx.x * digs + d] = 0;
  }
}

// One pass.  The first (tok given) takes the tokens and counts the high digit
// of each place it fills; the second takes the first's result.  Where a
// workgroup's elements of a digit go follows from the counts alone: all
// smaller digits, then this digit in earlier workgroups.
extern "C" __global__ __launch_bounds__(CHUNK) void hf_vocab_sort_pass(
    const int32_t* tok, const int* key, const int* pos, int T, int V, int bits,
    const unsigned* hist, unsigned* hist2, int* okey, int* opos, int blocks, Fill fill,
    VocabState* st) {
  if ((int)blockIdx.x >= blocks) {
    fill_rows(fill, blockIdx.x - blocks, gridDim.x - blocks);
    return;
  }
  __shared__ unsigned base[MAXDIG], mine[MAXDIG], tmp[16];
  const int digs = 1 << bits, t = blockIdx.x * CHUNK + threadIdx.x;
  for (int d = threadIdx.x; d < digs; d += CHUNK) base[d] = mine[d] = 0;
  __syncthreads();
  // every thread sums a digit over a share of the workgroups
  const int groups = max(1, CHUNK / digs);
  for (int i = threadIdx.x; i < digs * groups; i += CHUNK) {
    const int d = i & (digs - 1);
    unsigned all = 0, before = 0;
#pragma unroll 8
    for (int b = i >> bits; b < blocks; b += groups) {
      const unsigned x = hist[(size_t)b * digs + d];
      before += b < (int)blockIdx.x ? x : 0u;
      all += x;
    }
    atomicAdd(&base[d], all);
    atomicAdd(&mine[d], before);
  }
  __syncthreads();
  scan_digits(base, digs, tmp);
  for (int d = threadIdx.x; d < digs; d += CHUNK) base[d] += mine[d];
  __syncthreads();
  const bool valid = t < T;
  int k = 0, p = t;
  if (valid) {
    k = tok ? key_of(tok, t, V, st) : key[t];
    if (!tok) p = pos[t];
  }
  const int shift = tok ? 0 : bits;
  const unsigned at = place(base, (k >> shift) & (digs - 1), valid, bits);
  if (valid) {
    okey[at] = k;
    opos[at] = p;
  }
  if (tok) {
    // one addition per wave for the lanes of one high digit and workgroup
    // (frequent tokens share theirs)
    const unsigned slot = (at / CHUNK) * digs + ((unsigned)k >> bits);
    const unsigned long long m =
        alike(__ballot(valid), slot, 32 - __clz((unsigned)(blocks * digs - 1) | 1u));
    if (valid && (m & ((1ull << (threadIdx.x & 63)) - 1)) == 0)
      atomicAdd(&hist2[slot], (unsigned)__popcll(m));
  }
}

// Both passes of up to 1,024 rows in the first workgroup.
extern "C" __global__ __launch_bounds__(CHUNK) void hf_vocab_sort_one(
    const int32_t* tok, int T, int V, int bits, int* okey, int* opos, Fill fill,
    VocabState* st) {
  if (blockIdx.x > 0) {
    fill_rows(fill, blockIdx.x - 1, gridDim.x - 1);
    return;
  }
  __shared__ unsigned base[MAXDIG], tmp[16];
  __shared__ int key[CHUNK], pos[CHUNK];
  const int digs = 1 << bits, t = threadIdx.x;
  const bool valid = t < T;
  int k = valid ? key_of(tok, t, V, st) : 0, p = t;
  for (int pass = 0; pass < 2; ++pass) {
    for (int d = t; d < digs; d += CHUNK) base[d] = 0;
    __syncthreads();
    const int d = (k >> (pass * bits)) & (digs - 1);
    if (valid) atomicAdd(&base[d], 1u);
    __syncthreads();
    scan_digits(base, digs, tmp);
    const unsigned at = place(base, d, valid, bits);
    if (valid) {
      key[at] = k;
      pos[at] = p;
    }
    __syncthreads();
    if (valid) {
      k = key[t];
      p = pos[t];
    }
    __syncthreads();
  }
  if (valid) {
    okey[t] = k;
    opos[t] = p;
  }
}

// --------------------------------------------------------------- gradient
namespace {
// Sorted places per run: 32, or 16 where that leaves compute units without a
// wave (10,007 rows x 768 in fp32: 17 -> 12 us)
constexpr int RUN_MIN = 16, RUN_MAX = 32;

template <class E, bool VEC>
__device__ __forceinline__ void emit(E* row, int strip, int lane, int D, float scale,
                                     int accumulate, float (&acc)[Strip<E, VEC>::EPC]) {
  using S = Strip<E, VEC>;
#pragma unroll
  for (int e = 0; e < S::EPC; ++e) acc[e] *= scale;
  if (accumulate) {
    float old[S::EPC];
    S::load(row, strip, lane, D, old);
#pragma unroll
    for (int e = 0; e < S::EPC; ++e) acc[e] += old[e];
  }
  S::template store<false>(row, strip, lane, D, acc);
}

// One run and strip.  part[2 run]: the sum of the token that began before the
// run (or fills it from its start and goes on); part[2 run + 1]: of the one
// that begins within it and goes on.
template <class E, bool VEC, bool STREAM>
__device__ __forceinline__ void runs_body(const int* key, const int* pos, int RUN, int T, int V,
                                          int D, int strips, float scale, const E* dout,
                                          long long ldd, float* part, E* dE, long long lde,
                                          int accumulate) {
  using S = Strip<E, VEC>;
  const int lane = threadIdx.x & 63;
  const long long unit = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int run = (int)(unit / strips), strip = (int)(unit % strips);
  const int a = run * RUN;
  if (a >= T) return;
  // lane l: place a - 1 + l
  const int at = a - 1 + lane;
  const int k = at >= 0 && at < T && lane < RUN + 2 ? key[at] : -1;
  const int p = at >= 0 && at < T && lane < RUN + 1 ? pos[at] : 0;
  // places of tokens in the run (masked ones come last)
  const int n = __popcll(__ballot(lane >= 1 && lane <= RUN && k >= 0 && k < V));
  float acc[S::EPC] = {};
  int head = n > 0 && __shfl(k, 1, 64) == __shfl(k, 0, 64);
  constexpr int U = 16;      // rows in flight
  for (int i0 = 0; i0 < n; i0 += U) {
    typename S::Raw v[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i0 + u < n)
        v[u] = S::template raw<STREAM>(
            dout + (size_t)__builtin_amdgcn_readlane(p, 1 + i0 + u) * ldd, strip, lane, D);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i0 + u >= n) break;
#pragma unroll
      for (int e = 0; e < S::EPC; ++e) acc[e] += to_f(v[u].v[e]);
      const int cur = __builtin_amdgcn_readlane(k, 1 + i0 + u);
      const int nxt = __builtin_amdgcn_readlane(k, 2 + i0 + u);
      const bool last = i0 + u + 1 == RUN;
      if (cur == nxt && !last) continue;
      // the token's places in this run end here
      if (head || cur == nxt) {
        float* o = part + (((size_t)2 * run + !head) * strips + strip) * S::COLS +
                   lane * S::EPC;
#pragma unroll
        for (int q = 0; q < S::EPC / 4; ++q)
          *(f32x4*)(o + 4 * q) = f32x4{acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]};
      } else {
        emit<E, VEC>(dE + (size_t)cur * lde, strip, lane, D, scale, accumulate, acc);
      }
      head = 0;
#pragma unroll
      for (int e = 0; e < S::EPC; ++e) acc[e] = 0.0f;
    }
  }
}

// Tokens that span runs, a strip of columns: each wave looks at one boundary
// between runs.  Where a token has its first one, the wave joins it if it spans
// few runs; tokens that span many are summed by the 4 waves together, a quarter
// of the runs each, the quarters in order.
template <class E, bool VEC>
__device__ __forceinline__ void join_body(const int* key, int RUN, int T, int V, int D, int strips,
                                          float scale, const float* part, E* dE, long long lde,
                                          int accumulate) {
  using S = Strip<E, VEC>;
  constexpr int LONG = 16;
  __shared__ float quarter[4][S::COLS];
  __shared__ int ends[4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, strip = blockIdx.y;
  const int runs = (T + RUN - 1) / RUN;
  // acc += the token's partial sums of the runs x0 .. x1; it begins in `run`,
  // whose second partial sum is its
  auto sum = [&](int run, int x0, int x1, float (&acc)[S::EPC]) {
    auto at = [&](int x) {
      const size_t slot = 2 * (size_t)x + (x == run);
      return part + (slot * strips + strip) * S::COLS + lane * S::EPC;
    };
    constexpr int U = 8, Q = S::EPC / 4;
    for (int x = x0; x < x1; x += U) {
      f32x4 w[U][Q];
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int q = 0; q < Q; ++q) w[u][q] = *(const f32x4*)(at(min(x + u, x1 - 1)) + 4 * q);
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (x + u < x1)
#pragma unroll
          for (int e = 0; e < S::EPC; ++e) acc[e] += w[u][e / 4][e % 4];
    }
  };
  int last = 0;              // past the last run that starts with the token
  {
    const int run = blockIdx.x * 4 + wave, end = (run + 1) * RUN;
    if (end < T) {
      const int k = key[end], k1 = key[end - 1], k0 = run > 0 ? key[end - 1 - RUN] : -1;
      if (k < V && k1 == k && k0 != k) {
        // 64 probes at a time (one after the other, a search among 4,096 runs
        // took longer than the sums)
        int lo = run + 2, hi = runs;
        while (lo < hi) {
          const int stride = (hi - lo + 63) / 64, i = lo + lane * stride;
          const int n = __popcll(__ballot(i < hi && key[min(i, runs - 1) * RUN] == k));
          hi = min(hi, lo + n * stride);
          lo = n ? lo + (n - 1) * stride + 1 : lo;
        }
        last = lo;
        if (last - run <= LONG) {
          float acc[S::EPC] = {};
          sum(run, run, last, acc);
          emit<E, VEC>(dE + (size_t)k * lde, strip, lane, D, scale, accumulate, acc);
          last = 0;
        }
      }
    }
  }
  if (lane == 0) ends[wave] = last;
  __syncthreads();
  for (int w = 0; w < 4; ++w) {
    const int run = blockIdx.x * 4 + w, lo = ends[w];
    if (!lo) continue;
    const int per = (lo - run + 3) / 4;
    float acc[S::EPC] = {};
    sum(run, min(run + wave * per, lo), min(run + (wave + 1) * per, lo), acc);
    __syncthreads();
#pragma unroll
    for (int e = 0; e < S::EPC; ++e) quarter[wave][e * 64 + lane] = acc[e];
    __syncthreads();
    if (wave) continue;
#pragma unroll
    for (int e = 0; e < S::EPC; ++e)
      acc[e] = ((quarter[0][e * 64 + lane] + quarter[1][e * 64 + lane]) +
                quarter[2][e * 64 + lane]) + quarter[3][e * 64 + lane];
    emit<E, VEC>(dE + (size_t)key[(run + 1) * RUN] * lde, strip, lane, D, scale, accumulate, acc);
  }
}
}  // namespace

// _s: dout past the caches, where it and dE do not fit the last-level one, and
// partial sums and dE stay in them (131,072 x 2,048 of bf16: 173 -> 126 us, and
// the join 26 -> 18; whole calls of 8,192 rows, 32,000 x 4,096: 86 -> 77; but
// 30,000 rows, 50,257 x 768 of fp32, 246 MB: 65 -> 75)
#define HF_EMBED_RUNS(SUF, E, VEC, STREAM)                                               \
  extern "C" __global__ __launch_bounds__(256) void hf_vocab_embed_runs_##SUF(           \
      const int* key, const int* pos, int RUN, int T, int V, int D, int strips, float scale, \
      const E* dout, long long ldd, float* part, E* dE, long long lde, int accumulate) { \
    runs_body<E, VEC, STREAM>(key, pos, RUN, T, V, D, strips, scale, dout, ldd, part, dE, \
                              lde, accumulate);                                          \
  }
#define HF_EMBED_JOIN(SUF, E, VEC)                                                       \
  extern "C" __global__ __launch_bounds__(256, 5) void hf_vocab_embed_join_##SUF(        \
      const int* key, int RUN, int T, int V, int D, int strips, float scale,             \
      const float* part, E* dE, long long lde, int accumulate) {                         \
    join_body<E, VEC>(key, RUN, T, V, D, strips, scale, part, dE, lde, accumulate);      \
  }
HF_EMBED_RUNS(f32, float, false, false)
HF_EMBED_RUNS(f32_v, float, true, false)
HF_EMBED_RUNS(f32_s, float, true, true)
HF_EMBED_RUNS(bf16, bf16_t, false, false)
HF_EMBED_RUNS(bf16_v, bf16_t, true, false)
HF_EMBED_RUNS(bf16_s, bf16_t, true, true)
HF_EMBED_JOIN(f32, float, false)
HF_EMBED_JOIN(f32_v, float, true)
HF_EMBED_JOIN(bf16, bf16_t, false)
HF_EMBED_JOIN(bf16_v, bf16_t, true)

// ------------------------------------------------------------- launchers
namespace {
inline dim3 grid_of(dim3 g) { return g; }
inline dim3 grid_of(long long g) { return dim3((unsigned)g); }
}  // namespace
#define HF_LAUNCH(NAME, K, GRID, BLOCK, ...)                                       \
  do {                                                                             \
    prof_begin(L, NAME);                                                           \
    hipExtLaunchKernelGGL(K, grid_of(GRID), dim3(BLOCK), 0, L.stream,     \
                          prof_a(L), prof_b(L), 0, __VA_ARGS__);                   \
    prof_end(L, NAME, 0.0, 0.0);                                                   \
  } while (0)

namespace {
// see Strip
inline bool chunks(int D, int es) {
  const int epc = 16 / es, over = D % (64 * epc);
  return D >= epc && (over == 0 || over >= epc);
}
inline int strips_of(int D, int es) { return (D + 1024 / es - 1) / (1024 / es); }
inline int digit_bits(int V) {
  int b = 1;
  while ((1ll << (2 * b)) < (long long)V + 1) ++b;
  return b;
}
}  // namespace

size_t vocab_sort_hist(long long T, int V) {
  return T <= CHUNK ? 0 : 2 * ((size_t)1 << digit_bits(V)) * (size_t)((T + CHUNK - 1) / CHUNK);
}
size_t vocab_sort_part(long long T, int D, int type) {
  const int es = type == VT_F32 ? 4 : 2;
  return 2 * (size_t)((T + RUN_MIN - 1) / RUN_MIN) * strips_of(D, es) * (1024 / es);
}

void vocab_embed(const Launch& L, int type, const void* E, long long lde, int V, int D,
                 const int32_t* tok, int T, float scale, void* out, long long ldo,
                 VocabState* st) {
  if (T < 1) return;
  const int es = type == VT_F32 ? 4 : 2, strips = strips_of(D, es);
  const bool vec = chunks(D, es);
  // (a launch has fewer than 2^32 work-items in x: 262,144 rows of 65,536 of fp32
  // are as many)
  constexpr long long MAX_X = 1 << 20;
  const long long groups = ((long long)T * strips + 3) / 4;
  const dim3 grid((unsigned)std::min(groups, MAX_X), (unsigned)((groups + MAX_X - 1) / MAX_X));
  // _s: much output does not take the place of frequent tokens' rows of E in the
  // caches (65,536 x 4,096 of bf16: with cold caches 179 -> 160 us, call after call
  // 182 -> 108); little stays for its reader
  const bool stream = (long long)T * D * es > L2_BYTES;
#define HF_EMB(SUF, E_T)                                                                   \
  HF_LAUNCH("hf_vocab_embed",                                                              \
            (vec && stream ? hf_vocab_embed_##SUF##_s                                      \
             : vec         ? hf_vocab_embed_##SUF##_v                                      \
                           : hf_vocab_embed_##SUF),                                        \
            grid, 256, (const E_T*)E, lde, V, D, tok, T, strips, scale, (E_T*)out, ldo, st)
  if (type == VT_F32) HF_EMB(f32, float);
  else HF_EMB(bf16, bf16_t);
#undef HF_EMB
}

void vocab_embed_grad(const Launch& L, int type, const int32_t* tok, int T, int V, int D,
                      float scale, const void* dout, long long ldd, void* dE, long long lde,
                      int accumulate, const VSort& s, VocabState* st) {
  const int es = type == VT_F32 ? 4 : 2, strips = strips_of(D, es), bits = digit_bits(V);
  const bool vec = chunks(D, es);
  // the rows to fill, in shares like the durations of the sort's launches
  const size_t row = (size_t)lde * es;
  const Fill all = {accumulate ? nullptr : (char*)dE, (long long)row, D * es, 0, 0};
  auto share = [&](double a, double b) {
    Fill f = all;
    f.v0 = (int)(a * V);
    f.v1 = b < 1.0 ? (int)(b * V) : V;
    return f;
  };
  // workgroups that fill: two per compute unit, or fewer for little
  const int fills =
      accumulate ? 0 : (int)std::min<long long>(512, ((long long)V * all.bytes >> 16) + 1);
  if (T <= CHUNK) {
    if (T > 0 || fills)
      HF_LAUNCH("hf_vocab_sort", hf_vocab_sort_one, 1 + fills, CHUNK, tok, T, V, bits, s.key,
                s.pos, share(0.0, 1.0), st);
  } else {
    const int blocks = (T + CHUNK - 1) / CHUNK;
    unsigned* h2 = s.hist + ((size_t)1 << bits) * blocks;
    HF_LAUNCH("hf_vocab_sort", hf_vocab_sort_hist, blocks + fills, CHUNK, tok, T, V, bits,
              s.hist, h2, blocks, share(0.0, 0.2), st);
    HF_LAUNCH("hf_vocab_sort", hf_vocab_sort_pass, blocks + fills, CHUNK, tok,
              (const int*)nullptr, (const int*)nullptr, T, V, bits, (const unsigned*)s.hist, h2,
              s.tkey, s.tpos, blocks, share(0.2, 0.6), st);
    HF_LAUNCH("hf_vocab_sort", hf_vocab_sort_pass, blocks + fills, CHUNK,
              (const int32_t*)nullptr, (const int*)s.tkey, (const int*)s.tpos, T, V, bits,
              (const unsigned*)h2, (unsigned*)nullptr, s.key, s.pos, blocks, share(0.6, 1.0),
              st);
  }
  if (T < 1) return;
  const int RUN = (long long)((T + RUN_MAX - 1) / RUN_MAX) * strips < 2048 ? RUN_MIN : RUN_MAX;
  const int runs = (T + RUN - 1) / RUN;
  const long long units = (long long)runs * strips;
  const bool stream = ((long long)T + V) * D * es > L3_BYTES;
#define HF_EG(SUF, E)                                                                         \
  do {                                                                                        \
    HF_LAUNCH("hf_vocab_embed_runs",                                                          \
              (vec && stream ? hf_vocab_embed_runs_##SUF##_s                                  \
               : vec         ? hf_vocab_embed_runs_##SUF##_v                                  \
                             : hf_vocab_embed_runs_##SUF),                                    \
              (units + 3) / 4, 256, (const int*)s.key, (const int*)s.pos, RUN, T, V, D, strips, \
              scale, (const E*)dout, ldd, s.part, (E*)dE, lde, accumulate);                   \
    if (runs > 1)                                                                             \
      HF_LAUNCH("hf_vocab_embed_join",                                                        \
                (vec ? hf_vocab_embed_join_##SUF##_v : hf_vocab_embed_join_##SUF),            \
                dim3((runs + 3) / 4, strips), 256, (const int*)s.key, RUN, T, V, D, strips, scale, \
                (const float*)s.part, (E*)dE, lde, accumulate);                               \
  } while (0)
  if (type == VT_F32) HF_EG(f32, float);
  else HF_EG(bf16, bf16_t);
#undef HF_EG
}

}  // namespace hfk
