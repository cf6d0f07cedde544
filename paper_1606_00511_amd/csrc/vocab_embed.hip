// Token embedding and its gradient.
//   forward   out_t = scale E[tok_t], zeros where the token is masked
//   gradient  dE_v = scale sum_{t: tok_t = v} dout_t, in token order, fp32
// Both are bound by memory: each row is read and written once.
//
// The gradient sorts the rows by token (stable, two radix passes), so that the
// rows of one token are consecutive and every row of dE is written by one
// workgroup, zeros included: no atomics on sums, the same bits every time.
// Runs of 64 sorted places that hold one token only are summed beforehand in
// parallel; a frequent token's row then adds those sums instead of its rows.
#include "vocab_internal.h"

namespace hfk {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ uint32_t f2bf(float f) {
  return __builtin_bit_cast(uint16_t, (__bf16)f);
}
__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(bf16_t v) { return __uint_as_float((uint32_t)v << 16); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(bf16_t* p, float v) { *p = (bf16_t)f2bf(v); }

constexpr int IGNORE = -100;

// A wave has EPC columns of a row per lane and strip: 16 consecutive bytes
// (VEC: rows 16-byte aligned and whole chunks), else single elements 64 apart.
template <class E, bool VEC>
struct Strip {
  static constexpr int EPC = 16 / (int)sizeof(E);
  static constexpr int COLS = 64 * EPC;
  __device__ static __forceinline__ int col(int strip, int lane, int e) {
    return strip * COLS + (VEC ? lane * EPC + e : e * 64 + lane);
  }
  __device__ static __forceinline__ void load(const E* row, int strip, int lane, int D,
                                              float (&v)[EPC]) {
    if constexpr (VEC) {
      E w[EPC] = {};
      if (col(strip, lane, 0) < D) *(u32x4*)w = *(const u32x4*)(row + col(strip, lane, 0));
#pragma unroll
      for (int e = 0; e < EPC; ++e) v[e] = to_f(w[e]);
    } else {
#pragma unroll
      for (int e = 0; e < EPC; ++e) {
        const int c = col(strip, lane, e);
        v[e] = c < D ? to_f(row[c]) : 0.0f;
      }
    }
  }
  __device__ static __forceinline__ void store(E* row, int strip, int lane, int D,
                                               const float (&v)[EPC]) {
    if constexpr (VEC) {
      E w[EPC];
#pragma unroll
      for (int e = 0; e < EPC; ++e) put(w + e, v[e]);
      if (col(strip, lane, 0) < D) *(u32x4*)(row + col(strip, lane, 0)) = *(u32x4*)w;
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
template <class E, bool VEC>
__device__ __forceinline__ void embed_body(const E* table, long long lde, int V, int D,
                                           const int32_t* tok, int T, int strips, float scale,
                                           E* out, long long ldo, VocabState* st) {
  using S = Strip<E, VEC>;
  const int lane = threadIdx.x & 63;
  const long long u = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
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
  S::store(out + (size_t)t * ldo, strip, lane, D, v);
}

}  // namespace

#define HF_EMBED(SUF, E, VEC)                                                            \
  extern "C" __global__ __launch_bounds__(256) void hf_vocab_embed_##SUF(                \
      const E* table, long long lde, int V, int D, const int32_t* tok, int T, int strips, \
      float scale, E* out, long long ldo, VocabState* st) {                              \
    embed_body<E, VEC>(table, lde, V, D, tok, T, strips, scale, out, ldo, st);           \
  }
HF_EMBED(f32, float, false)
HF_EMBED(f32_v, float, true)
HF_EMBED(bf16, bf16_t, false)
HF_EMBED(bf16_v, bf16_t, true)

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

// The place of each thread's element among the elements of its digit: `base`
// holds where each digit's next element goes.  The waves take their turns in
// order, so that equal digits keep their order.
__device__ __forceinline__ unsigned place(unsigned* base, int d, bool valid, int bits) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  unsigned long long same = __ballot(valid);
  for (int b = 0; b < bits; ++b) {
    const unsigned long long m = __ballot((d >> b) & 1);
    same &= ((d >> b) & 1) ? m : ~m;
  }
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
    const int32_t* tok, int T, int V, int bits, unsigned* hist, unsigned* hist2,
    VocabState* st) {
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
    const unsigned* hist, unsigned* hist2, int* okey, int* opos, VocabState* st) {
  __shared__ unsigned base[MAXDIG], mine[MAXDIG], tmp[16];
  const int digs = 1 << bits, blocks = gridDim.x, t = blockIdx.x * CHUNK + threadIdx.x;
  for (int d = threadIdx.x; d < digs; d += CHUNK) base[d] = mine[d] = 0;
  __syncthreads();
  // every thread sums a digit over a share of the workgroups
  const int groups = max(1, CHUNK / digs);
  for (int i = threadIdx.x; i < digs * groups; i += CHUNK) {
    const int d = i & (digs - 1);
    unsigned all = 0, before = 0;
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
    if (tok) atomicAdd(&hist2[(size_t)(at / CHUNK) * digs + (k >> bits)], 1u);
  }
}

// Both passes of up to 1,024 rows in one workgroup.
extern "C" __global__ __launch_bounds__(CHUNK) void hf_vocab_sort_one(
    const int32_t* tok, int T, int V, int bits, int* okey, int* opos, VocabState* st) {
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
constexpr int RUN = 64;      // sorted places per chunk
constexpr int VROWS = 8;     // rows of dE per workgroup

// acc += rows pos[a .. b) of dout
template <class E, bool VEC>
__device__ __forceinline__ void add_rows(const E* dout, long long ldd, const int* pos, int a,
                                         int b, int strip, int lane, int D,
                                         float (&acc)[Strip<E, VEC>::EPC]) {
  using S = Strip<E, VEC>;
  constexpr int U = 8;
  int i = a;
  for (; i + U <= b; i += U) {
    float v[U][S::EPC];
#pragma unroll
    for (int u = 0; u < U; ++u)
      S::load(dout + (size_t)__builtin_amdgcn_readfirstlane(pos[i + u]) * ldd, strip, lane, D,
              v[u]);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < S::EPC; ++e) acc[e] += v[u][e];
  }
  for (; i < b; ++i) {
    float v[S::EPC];
    S::load(dout + (size_t)__builtin_amdgcn_readfirstlane(pos[i]) * ldd, strip, lane, D, v);
#pragma unroll
    for (int e = 0; e < S::EPC; ++e) acc[e] += v[e];
  }
}

// part[c][col] = sum of the chunk's rows, where all of them are one token's;
// col as the lane has it, strip by strip
template <class E, bool VEC>
__device__ __forceinline__ void chunk_body(const int* key, const int* pos, int V, int D,
                                           int strips, const E* dout, long long ldd,
                                           float* part) {
  using S = Strip<E, VEC>;
  const int c = blockIdx.x, a = c * RUN;
  const int k = key[a];
  if (k >= V || key[a + RUN - 1] != k) return;
  const int lane = threadIdx.x & 63;
  for (int strip = threadIdx.x >> 6; strip < strips; strip += 4) {
    float acc[S::EPC] = {};
    add_rows<E, VEC>(dout, ldd, pos, a, a + RUN, strip, lane, D, acc);
    float* p = part + ((size_t)c * strips + strip) * S::COLS;
#pragma unroll
    for (int e = 0; e < S::EPC; ++e) p[e * 64 + lane] = acc[e];
  }
}

template <class E, bool VEC>
__device__ __forceinline__ void grad_body(const int* key, const int* pos, int T, int V, int D,
                                          int strips, float scale, const E* dout, long long ldd,
                                          const float* part, E* dE, long long lde,
                                          int accumulate) {
  using S = Strip<E, VEC>;
  __shared__ int lb[VROWS + 1];
  const int v0 = blockIdx.x * VROWS, tid = threadIdx.x, lane = tid & 63;
  if (tid <= VROWS) {
    // first place whose token is not below v
    const int v = v0 + tid;
    int lo = 0, hi = T;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (key[mid] < v) lo = mid + 1;
      else hi = mid;
    }
    lb[tid] = lo;
  }
  __syncthreads();
  for (int u = tid >> 6; u < VROWS * strips; u += 4) {
    const int i = u / strips, strip = u % strips, v = v0 + i;
    if (v >= V) return;
    const int a = __builtin_amdgcn_readfirstlane(lb[i]);
    const int b = __builtin_amdgcn_readfirstlane(lb[i + 1]);
    if (a == b && accumulate) continue;
    E* row = dE + (size_t)v * lde;
    float acc[S::EPC] = {};
    const int c0 = (a + RUN - 1) / RUN, c1 = b / RUN;
    if (c0 < c1) {
      add_rows<E, VEC>(dout, ldd, pos, a, c0 * RUN, strip, lane, D, acc);
      int c = c0;
      constexpr int U = 4;
      for (; c + U <= c1; c += U) {
        float w[U][S::EPC];
#pragma unroll
        for (int x = 0; x < U; ++x)
#pragma unroll
          for (int e = 0; e < S::EPC; ++e)
            w[x][e] = part[((size_t)(c + x) * strips + strip) * S::COLS + e * 64 + lane];
#pragma unroll
        for (int x = 0; x < U; ++x)
#pragma unroll
          for (int e = 0; e < S::EPC; ++e) acc[e] += w[x][e];
      }
      for (; c < c1; ++c)
#pragma unroll
        for (int e = 0; e < S::EPC; ++e)
          acc[e] += part[((size_t)c * strips + strip) * S::COLS + e * 64 + lane];
      add_rows<E, VEC>(dout, ldd, pos, c1 * RUN, b, strip, lane, D, acc);
    } else {
      add_rows<E, VEC>(dout, ldd, pos, a, b, strip, lane, D, acc);
    }
#pragma unroll
    for (int e = 0; e < S::EPC; ++e) acc[e] *= scale;
    if (accumulate) {
      float old[S::EPC];
      S::load(row, strip, lane, D, old);
#pragma unroll
      for (int e = 0; e < S::EPC; ++e) acc[e] += old[e];
    }
    S::store(row, strip, lane, D, acc);
  }
}
}  // namespace

#define HF_EMBED_GRAD(SUF, E, VEC)                                                          \
  extern "C" __global__ __launch_bounds__(256) void hf_vocab_embed_chunk_##SUF(             \
      const int* key, const int* pos, int V, int D, int strips, const E* dout,              \
      long long ldd, float* part) {                                                         \
    chunk_body<E, VEC>(key, pos, V, D, strips, dout, ldd, part);                            \
  }                                                                                         \
  extern "C" __global__ __launch_bounds__(256) void hf_vocab_embed_grad_##SUF(              \
      const int* key, const int* pos, int T, int V, int D, int strips, float scale,         \
      const E* dout, long long ldd, const float* part, E* dE, long long lde,                \
      int accumulate) {                                                                     \
    grad_body<E, VEC>(key, pos, T, V, D, strips, scale, dout, ldd, part, dE, lde, accumulate); \
  }
HF_EMBED_GRAD(f32, float, false)
HF_EMBED_GRAD(f32_v, float, true)
HF_EMBED_GRAD(bf16, bf16_t, false)
HF_EMBED_GRAD(bf16_v, bf16_t, true)

// ------------------------------------------------------------- launchers
#define HF_LAUNCH(NAME, K, GRID, BLOCK, ...)                                       \
  do {                                                                             \
    prof_begin(L, NAME);                                                           \
    hipExtLaunchKernelGGL(K, dim3((unsigned)(GRID)), dim3(BLOCK), 0, L.stream,     \
                          prof_a(L), prof_b(L), 0, __VA_ARGS__);                   \
    prof_end(L, NAME, 0.0, 0.0);                                                   \
  } while (0)

namespace {
// rows take whole 16-byte chunks
inline bool vec16(const void* p, long long ld, int D, int es) {
  return ((uintptr_t)p & 15) == 0 && (ld * es) % 16 == 0 && ((long long)D * es) % 16 == 0;
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
  return (size_t)(T / RUN) * strips_of(D, es) * (1024 / es);
}

void vocab_embed(const Launch& L, int type, const void* E, long long lde, int V, int D,
                 const int32_t* tok, int T, float scale, void* out, long long ldo,
                 VocabState* st) {
  if (T < 1) return;
  const int es = type == VT_F32 ? 4 : 2, strips = strips_of(D, es);
  const bool vec = vec16(E, lde, D, es) && vec16(out, ldo, D, es);
  const long long grid = ((long long)T * strips + 3) / 4;
  if (type == VT_F32)
    HF_LAUNCH("hf_vocab_embed", (vec ? hf_vocab_embed_f32_v : hf_vocab_embed_f32), grid, 256,
              (const float*)E, lde, V, D, tok, T, strips, scale, (float*)out, ldo, st);
  else
    HF_LAUNCH("hf_vocab_embed", (vec ? hf_vocab_embed_bf16_v : hf_vocab_embed_bf16), grid, 256,
              (const bf16_t*)E, lde, V, D, tok, T, strips, scale, (bf16_t*)out, ldo, st);
}

void vocab_embed_grad(const Launch& L, int type, const int32_t* tok, int T, int V, int D,
                      float scale, const void* dout, long long ldd, void* dE, long long lde,
                      int accumulate, const VSort& s, VocabState* st) {
  const int es = type == VT_F32 ? 4 : 2, strips = strips_of(D, es), bits = digit_bits(V);
  const bool vec = vec16(dout, ldd, D, es) && vec16(dE, lde, D, es);
  if (T > 0 && T <= CHUNK) {
    HF_LAUNCH("hf_vocab_sort", hf_vocab_sort_one, 1, CHUNK, tok, T, V, bits, s.key, s.pos, st);
  } else if (T > 0) {
    const int blocks = (T + CHUNK - 1) / CHUNK;
    unsigned* h2 = s.hist + ((size_t)1 << bits) * blocks;
    HF_LAUNCH("hf_vocab_sort", hf_vocab_sort_hist, blocks, CHUNK, tok, T, V, bits, s.hist, h2,
              st);
    HF_LAUNCH("hf_vocab_sort", hf_vocab_sort_pass, blocks, CHUNK, tok, (const int*)nullptr,
              (const int*)nullptr, T, V, bits, (const unsigned*)s.hist, h2, s.tkey, s.tpos, st);
    HF_LAUNCH("hf_vocab_sort", hf_vocab_sort_pass, blocks, CHUNK, (const int32_t*)nullptr,
              (const int*)s.tkey, (const int*)s.tpos, T, V, bits, (const unsigned*)h2,
              (unsigned*)nullptr, s.key, s.pos, st);
  }
  const int chunks = T / RUN, grid = (V + VROWS - 1) / VROWS;
#define HF_EG(SUF, E)                                                                        \
  do {                                                                                       \
    if (chunks > 0)                                                                          \
      HF_LAUNCH("hf_vocab_embed_chunk",                                                      \
                (vec ? hf_vocab_embed_chunk_##SUF##_v : hf_vocab_embed_chunk_##SUF), chunks, \
                256, (const int*)s.key, (const int*)s.pos, V, D, strips, (const E*)dout, ldd, \
                s.part);                                                                     \
    HF_LAUNCH("hf_vocab_embed_grad",                                                         \
              (vec ? hf_vocab_embed_grad_##SUF##_v : hf_vocab_embed_grad_##SUF), grid, 256,  \
              (const int*)s.key, (const int*)s.pos, T, V, D, strips, scale, (const E*)dout,  \
              ldd, (const float*)s.part, (E*)dE, lde, accumulate);                           \
  } while (0)
  if (type == VT_F32) HF_EG(f32, float);
  else HF_EG(bf16, bf16_t);
#undef HF_EG
}

}  // namespace hfk
