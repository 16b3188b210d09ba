// Log-prob, entropy and log-sum-exp of tokens from hidden states and the head's weights, and the gradient
// (formulas: include/rl_linear_logprob.h).
//
// Matrix-core bound from some hundred rows on (2 rows x hidden x vocab operations a product; one forward, one to recompute, two for
// the gradients), below that bound by reading the weights.  All four products are rlda_tile.h's, with the larger of the two
// free dimensions' elements along the registers (m) so that what follows a product stays inside a lane:
//   forward    m = vocabulary, n = tokens: a lane has 16 logits of a token per block, reduces them to (max, sum, sum of
//              e x distance from the max) in base 2, halves and wavefronts meet once per tile, tiles in a second kernel
//   recompute  the same product, then dz in bf16 to scratch [token][vocabulary of the piece]
//   dhidden    m = hidden, k = vocabulary of the piece: weight rows are read transposed from LDS; few output tiles, so k
//              is cut into splits with sums of their own (fp32), which a last kernel adds in order
//   dweight    m = hidden, n = vocabulary, k = tokens: both operands transposed
// Scratch is zero where a token or a column does not exist, and so is, in LDS, what a tile of weights has behind its last column or row: no product needs a mask.
//
// Weights that mask a token are infinite or NaN, and its dz, which is 0, would make NaN of them in dhidden.  A logit that is not finite says that there may
// be some (hidden states that add anything are finite, unless they mask their row's every logit): the recomputation then raises a flag, and dhidden's
// product reads the weights' infinities and NaN as zeros (50 NaN rows: recompute and dhidden of 2048 x 3584 x 151936 4.19 -> 4.53 ms, 333 x 896 x 50001 108 -> 135 us).
// Only a masked token that was sampled has a dz; its infinities are added at the end.
//
// dz rounded to bf16 is off by the roundings of its few large elements; over many tokens they average out beside the result's own, over a
// few they need not (2 tokens: dweight 2.4e-3 of its norm off against 1.6e-3).  Up to 32 tokens, whose tiles of 64 are half empty, the second half
// holds what the first one's rounding left over: the products take it along as tokens of their own.
//
// Measured: 4096 tokens x 3584 x 151936 forward 3.83 ms (1.16 Pflop/s, 82 % of the library's bare product); 2048 tokens with gradient 8.18 ms: forward
// 1.96, recompute 2.2, dhidden 2.0, dweight 1.9; 333 x 896 x 50001 forward 44 us, recompute 50, dhidden 40, dweight 44; 16 x 2048 x 151936, the weights at 4.4 to 5.5 TB/s:
// 114, 140, 113, 125.
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <atomic>
#include <type_traits>

#include "../../include/rl_linear_logprob.h"
#include "rlda_tile.h"

namespace {

using namespace rlda;

constexpr float LN2 = 0.69314718055994531f, LOG2E = 1.4426950408889634f;
constexpr float MASKED = -1e30f;                            // stands for a masked logit: a finite number, so that 0 * MASKED is 0

// Workgroups along x of a launch, a multiple of 8; more go along another dimension.  A dimension of a grid holds fewer than 2^32 threads, and a launch of
// more is accepted and runs in part.
constexpr int GRID_X = 1 << 21;

struct Shape {
  int N, V, H;
  int tiles_m, tiles_n;
};

// Tile of a workgroup.  Workgroups go round the 8 dies; each die gets a contiguous run of the tiles, in which 8 tiles along n
// come before the next along m, so that the 32 workgroups of a die read few different rows at a time.
__device__ __forceinline__ bool place(const Shape& s, int& tm, int& tn) {
  const int total = s.tiles_m * s.tiles_n, per = (total + 7) / 8, b = (int)(blockIdx.y * GRID_X + blockIdx.x);
  const int t = (b & 7) * per + (b >> 3);
  if (b >> 3 >= per || t >= total) return false;
  const int group = t / (8 * s.tiles_m), first = group * 8, width = min(8, s.tiles_n - first), in = t - group * 8 * s.tiles_m;
  tm = in / width;
  tn = first + in % width;
  return true;
}
dim3 grid_of(int tiles) {
  const int n = (tiles + 7) / 8 * 8;
  return dim3(n < GRID_X ? n : GRID_X, (n + GRID_X - 1) / GRID_X);
}

// sums over the logits of a token, in base 2: m = max, s = sum 2^(z - m), t = sum 2^(z - m) (z - m)
struct Acc { float m, s, t; };
__device__ __forceinline__ Acc merge(const Acc& x, const Acc& y) {
  const float m = fmaxf(x.m, y.m), dx = x.m - m, dy = y.m - m;
  const float cx = __builtin_amdgcn_exp2f(dx), cy = __builtin_amdgcn_exp2f(dy);
  return Acc{m, x.s * cx + y.s * cy, cx * fmaf(x.s, dx, x.t) + cy * fmaf(y.s, dy, y.t)};
}

struct ForwardParams {
  Shape s;
  const void* hidden; const void* weight; const int32_t* ids;
  int64_t hs, ws;                                           // elements between rows
  float k2;                                                 // inv_temperature * log2 e
  float4* part;                                             // [tiles_m][N]: m, s, t of a tile
  float* zy;                                                // [N] base-2 logit of the sampled token
};

template <typename T>
__device__ __forceinline__ void logits(const ForwardParams& P, int tm, int tn, uint32_t lds, f32x16 (&acc)[T::MT][T::NT]) {
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  typename T::OA a;
  typename T::OB b;
  a.init(P.weight, P.ws, (int64_t)tm * T::BM, P.s.V, wv, lane);
  b.init(P.hidden, P.hs, (int64_t)tn * T::BN, P.s.N, wv, lane);
  const int nk = (P.s.H + T::BK - 1) / T::BK, tail = P.s.H % T::BK;
  T::run(a, b, 0, nk, tail ? nk - 1 : -1, tail / 8, lds, acc);
}

template <typename T>
__global__ void __launch_bounds__(T::THREADS, T::THREADS == 512 ? 2 : 4) linear_logprob_kernel(const ForwardParams P) {
  extern __shared__ __attribute__((aligned(1024))) char lds_all[];
  int tm, tn;
  if (!place(P.s, tm, tn)) return;
  const uint32_t lds = (uint32_t)(uintptr_t)RLDA_AS3(char, lds_all);
  f32x16 acc[T::MT][T::NT];
  logits<T>(P, tm, tn, lds, acc);
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wv % T::WM, wn = wv / T::WM;
  const int v0 = tm * T::BM + wm * T::MT * 32 + 4 * (lane >> 5);
  float4* const red = reinterpret_cast<float4*>(lds_all);   // [WM][BN]
  const bool whole = (tm + 1) * T::BM <= P.s.V;
#pragma unroll
  for (int j = 0; j < T::NT; ++j) {
    const int nl = (wn * T::NT + j) * 32 + (lane & 31), n = tn * T::BN + nl;
    const int y = n < P.s.N ? P.ids[n] : -1;
    Acc A{MASKED, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < T::MT; ++i)
#pragma unroll
      for (int x = 0; x < 16; ++x) {
        float z = fmaxf(acc[i][j][x] * P.k2, MASKED);
        if (!whole && v0 + 32 * i + 8 * (x >> 2) + (x & 3) >= P.s.V) z = MASKED;
        acc[i][j][x] = z;
        A.m = fmaxf(A.m, z);
      }
#pragma unroll
    for (int i = 0; i < T::MT; ++i)
#pragma unroll
      for (int x = 0; x < 16; ++x) {
        const float d = acc[i][j][x] - A.m, e = __builtin_amdgcn_exp2f(d);
        A.s += e;
        A.t = fmaf(e, d, A.t);
      }
    if (__any(y >= v0 && y < v0 + T::MT * 32)) {
#pragma unroll
      for (int i = 0; i < T::MT; ++i)
#pragma unroll
        for (int x = 0; x < 16; ++x)
          if (v0 + 32 * i + 8 * (x >> 2) + (x & 3) == y) P.zy[n] = acc[i][j][x];
    }
    A = merge(A, Acc{__shfl_xor(A.m, 32, 64), __shfl_xor(A.s, 32, 64), __shfl_xor(A.t, 32, 64)});
    if (lane < 32) red[wm * T::BN + nl] = make_float4(A.m, A.s, A.t, 0.f);
  }
  __syncthreads();
  for (int nl = threadIdx.x; nl < T::BN; nl += T::THREADS) {
    const int n = tn * T::BN + nl;
    if (n >= P.s.N) break;
    float4 v = red[nl];
    Acc A{v.x, v.y, v.z};
#pragma unroll
    for (int w = 1; w < T::WM; ++w) {
      v = red[w * T::BN + nl];
      A = merge(A, Acc{v.x, v.y, v.z});
    }
    P.part[(size_t)tm * P.s.N + n] = make_float4(A.m, A.s, A.t, 0.f);
  }
}

// the tiles of TOKENS tokens, 256 / TOKENS threads to a token
template <int TOKENS>
__global__ void __launch_bounds__(256) linear_logprob_merge_kernel(const ForwardParams P, float* logprob, float* lse, float* entropy) {
  constexpr int LANES = 256 / TOKENS;
  __shared__ Acc red[LANES][TOKENS];
  const int nl = threadIdx.x % TOKENS, part = threadIdx.x / TOKENS, n = blockIdx.x * TOKENS + nl;
  Acc A{MASKED, 0.f, 0.f};
  if (n < P.s.N)
#pragma unroll 4
    for (int t = part; t < P.s.tiles_m; t += LANES) {
      const float4 v = P.part[(size_t)t * P.s.N + n];
      A = merge(A, Acc{v.x, v.y, v.z});
    }
  red[part][nl] = A;
  for (int w = LANES / 2; w > 0; w >>= 1) {
    __syncthreads();
    if (part < w) red[part][nl] = A = merge(A, red[part + w][nl]);
  }
  if (part > 0 || n >= P.s.N) return;
  const bool dead = A.m <= MASKED;
  const float l2 = __log2f(A.s), lse2 = A.m + l2;
  if (lse) lse[n] = dead ? -INFINITY : lse2 * LN2;
  if (entropy) entropy[n] = dead ? NAN : (l2 - A.t / A.s) * LN2;
  if (logprob) {
    const int y = P.ids[n];
    float lp = 0.f;
    if (y >= P.s.V) lp = NAN;
    else if (y >= 0) {
      const float z = P.zy[n];
      lp = z <= MASKED && l2 == l2 ? -INFINITY : (z - A.m - l2) * LN2;                 // a logit of +inf leaves no distribution, for a masked token either
    }
    logprob[n] = lp;
  }
}

// what the epilogue of the recomputed product needs of a token: lse (base 2), g_logprob, g_entropy, entropy; zeros in g and a
// huge lse where it adds nothing
struct BackwardParams {
  ForwardParams f;                                          // hidden: the copy below
  const float4* token;                                      // [N64]
  __bf16* dz;                                               // [N64][ld]
  int64_t ld;
  int v0, v1;                                               // the piece
  float inv_t;
  bool twice;                                               // rows n + 32 of dz: what rounding left of rows n
  int* odd;                                                 // raised where a logit is not finite
};

// rows of hidden states that add something, zeros for the others and up to whole k-steps in both directions
__global__ void __launch_bounds__(256) linear_logprob_prepare_kernel(const char* hidden, int64_t hs, int N, int H, int V, int N64, int H64,
    const int32_t* ids, const float* lse, const float* entropy, const float* gl, const float* ge, char* copy, float4* token, bool twice,
    int* odd) {
  const int row = (int)(blockIdx.y * GRID_X + blockIdx.x), n = twice ? row & 31 : row;                       // twice: rows n + 32 again
  if (row >= N64) return;
  bool live = n < N;
  if (token) {
    if (row == 0 && threadIdx.x == 0) *odd = 0;
    float g = 0.f, e = 0.f, l = -INFINITY, ent = 0.f;
    if (live) {
      const int y = ids[n];
      l = lse[n];
      if (y >= 0 && y < V) g = gl[n];
      if (ge) { e = ge[n]; ent = entropy[n]; }
    }
    live = (g != 0.f || e != 0.f) && l != -INFINITY;        // NaN: a row with a logit of +inf; it passes on
    if (threadIdx.x < 4) {
      const int x = threadIdx.x;
      reinterpret_cast<float*>(token + row)[x] = live ? (x == 0 ? l * LOG2E : x == 1 ? g : x == 2 ? e : ent) : (x == 0 ? 1e30f : 0.f);
    }
  }
  for (int c = threadIdx.x; c < H64 / 8; c += 256) {
    uint4 v = make_uint4(0, 0, 0, 0);
    if (live && c < H / 8) v = *reinterpret_cast<const uint4*>(hidden + ((size_t)n * hs + c * 8) * 2);
    reinterpret_cast<uint4*>(copy)[(size_t)row * (H64 / 8) + c] = v;
  }
}

typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

template <typename T>
__global__ void __launch_bounds__(T::THREADS, T::THREADS == 512 ? 2 : 4) linear_logprob_dz_kernel(const BackwardParams P) {
  extern __shared__ __attribute__((aligned(1024))) char lds_all[];
  int tm, tn;
  if (!place(P.f.s, tm, tn)) return;
  f32x16 acc[T::MT][T::NT];
  logits<T>(P.f, tm, tn, (uint32_t)(uintptr_t)RLDA_AS3(char, lds_all), acc);
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wv % T::WM, wn = wv / T::WM;
  const int vl = tm * T::BM + wm * T::MT * 32 + 4 * (lane >> 5);                       // in the piece, whose rows f.weight starts at
  const int V = P.v1 - P.v0;
  const int N64 = (P.f.s.N + 63) / 64 * 64;
  float odd = 0.f;
#pragma unroll
  for (int j = 0; j < T::NT; ++j)
#pragma unroll
    for (int i = 0; i < T::MT; ++i)
#pragma unroll
      for (int x = 0; x < 16; ++x) odd = fmaf(acc[i][j][x], 0.f, odd);
  if (odd != 0.f) *P.odd = 1;
#pragma unroll
  for (int j = 0; j < T::NT; ++j) {
    const int n = tn * T::BN + (wn * T::NT + j) * 32 + (lane & 31);
    if (n >= N64 || (P.twice && j > 0)) continue;           // (tiles of 64 tokens: one wavefront along n)
    const float4 tk = P.token[n];
    const int y = n < P.f.s.N ? P.f.ids[n] - P.v0 : -1;
    __bf16* const row = P.dz + (size_t)n * P.ld;
#pragma unroll
    for (int i = 0; i < T::MT; ++i)
#pragma unroll
      for (int x4 = 0; x4 < 4; ++x4) {
        bf16x4 out, rest;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const int v = vl + 32 * i + 8 * x4 + x;
          const float lp2 = fmaxf(acc[i][j][4 * x4 + x] * P.f.k2, MASKED) - tk.x, p = __builtin_amdgcn_exp2f(lp2);
          float dz = -p * fmaf(tk.z, fmaf(lp2, LN2, tk.w), tk.y);
          if (v == y) dz += tk.y;
          dz = v < V ? dz * P.inv_t : 0.f;
          out[x] = (__bf16)dz;
          rest[x] = (__bf16)(dz - (float)out[x]);
        }
        *reinterpret_cast<bf16x4*>(row + vl + 32 * i + 8 * x4) = out;
        if (P.twice) *reinterpret_cast<bf16x4*>(row + 32 * P.ld + vl + 32 * i + 8 * x4) = rest;
      }
  }
}

struct DhiddenParams {
  int tiles_m, tiles_n, splits;
  const void* weight; int64_t ws;                           // the piece's rows
  int V, H, N64;                                            // rows of the piece
  const __bf16* dz; int64_t ld;
  float* sum;                                               // [splits][N64][H]
  int first;                                                // the first piece: written, not added to
  const int* odd;
};

template <typename T>
__global__ void __launch_bounds__(T::THREADS, T::THREADS == 512 ? 2 : 4) linear_logprob_dhidden_kernel(const DhiddenParams P) {
  extern __shared__ __attribute__((aligned(1024))) char lds_all[];
  const int split = blockIdx.x % P.splits, t = blockIdx.x / P.splits, tm = t % P.tiles_m, tn = t / P.tiles_m;
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wv % T::WM, wn = wv / T::WM;
  typename T::OA a;
  typename T::OB b;
  a.init(P.weight, P.ws, (int64_t)tm * T::BM, P.H, wv, lane);
  b.init(P.dz, P.ld, (int64_t)tn * T::BN, P.N64, wv, lane);
  const int nk = (P.V + T::BK - 1) / T::BK, tail = P.V % T::BK;
  const int k0 = (int)((int64_t)nk * split / P.splits), k1 = (int)((int64_t)nk * (split + 1) / P.splits);
  f32x16 acc[T::MT][T::NT];
  T::template run<true>(a, b, k0, k1, tail ? nk - 1 : -1, tail, (uint32_t)(uintptr_t)RLDA_AS3(char, lds_all), acc, *P.odd != 0);
#pragma unroll
  for (int j = 0; j < T::NT; ++j) {
    const int n = tn * T::BN + (wn * T::NT + j) * 32 + (lane & 31);
    if (n >= P.N64) continue;
#pragma unroll
    for (int i = 0; i < T::MT; ++i)
#pragma unroll
      for (int x4 = 0; x4 < 4; ++x4) {
        const int h = tm * T::BM + (wm * T::MT + i) * 32 + 8 * x4 + 4 * (lane >> 5);
        if (h >= P.H) continue;
        float4* const p = reinterpret_cast<float4*>(P.sum + ((size_t)split * P.N64 + n) * P.H + h);
        float4 v = make_float4(acc[i][j][4 * x4], acc[i][j][4 * x4 + 1], acc[i][j][4 * x4 + 2], acc[i][j][4 * x4 + 3]);
        if (!P.first) {
          const float4 o = *p;
          v.x += o.x; v.y += o.y; v.z += o.z; v.w += o.w;
        }
        *p = v;
      }
  }
}

// The splits' sums, rounded.  LANES threads share the slabs of four columns, in an order of their own that never changes: many slabs are those of few
// tokens, whose sums would else be one long chain of loads (16 tokens, 2048 columns: 115 -> 7 us).
template <int LANES>
__global__ void __launch_bounds__(256) linear_logprob_round_kernel(const float* sum, int splits, int64_t slab, int N, int H, __bf16* out, int64_t stride, bool twice,
    const int* odd, const __bf16* weight, int64_t ws, int V, const int32_t* ids, const float4* token, float inv_t) {
  __shared__ float4 part[256];
  constexpr int COLS = 256 / LANES;
  const int n = (int)(blockIdx.z * GRID_X + blockIdx.x);
  if (n >= N) return;
  const int col = threadIdx.x % COLS, lane = threadIdx.x / COLS, h = (blockIdx.y * COLS + col) * 4;
  float4 v{0.f, 0.f, 0.f, 0.f};
  if (h < H) {
    const float* p = sum + (size_t)n * H + h;
    for (int s = lane; s < splits; s += LANES) {
      const float4 o = *reinterpret_cast<const float4*>(p + s * slab);
      v.x += o.x; v.y += o.y; v.z += o.z; v.w += o.w;
      if (twice) {
        const float4 r = *reinterpret_cast<const float4*>(p + s * slab + (size_t)32 * H);
        v.x += r.x; v.y += r.y; v.z += r.z; v.w += r.w;
      }
    }
  }
  if constexpr (LANES > 1) {
    part[threadIdx.x] = v;
    __syncthreads();
    if (lane > 0) return;
#pragma unroll
    for (int s = 1; s < LANES; ++s) {
      const float4 o = part[s * COLS + col];
      v.x += o.x; v.y += o.y; v.z += o.z; v.w += o.w;
    }
  }
  if (h >= H) return;
  const int y = ids[n];
  if (*odd && y >= 0 && y < V && token[n].y != 0.f) {       // what dhidden's product left out: infinite weights of a masked token that was sampled
    const bf16x4 w = *reinterpret_cast<const bf16x4*>(weight + (size_t)y * ws + h);
    float* const to[4] = {&v.x, &v.y, &v.z, &v.w};
#pragma unroll
    for (int x = 0; x < 4; ++x)
      if (!(fabsf((float)w[x]) < INFINITY)) *to[x] += inv_t * token[n].y * (float)w[x];
  }
  *reinterpret_cast<bf16x4*>(out + (size_t)n * stride + h) = bf16x4{(__bf16)v.x, (__bf16)v.y, (__bf16)v.z, (__bf16)v.w};
}

struct DweightParams {
  Shape s;                                                  // N: N64; V: rows of the piece
  const void* hidden; int64_t hs;
  const __bf16* dz; int64_t ld;
  __bf16* out; int64_t stride;                              // the piece's rows
  bool past;                                                // stores go past the caches
};

template <typename T>
__global__ void __launch_bounds__(T::THREADS, 2) linear_logprob_dweight_kernel(const DweightParams P) {
  extern __shared__ __attribute__((aligned(1024))) char lds_all[];
  int tm, tn;
  if (!place(P.s, tm, tn)) return;
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wv % T::WM, wn = wv / T::WM;
  typename T::OA a;
  typename T::OB b;
  a.init(P.hidden, P.hs, (int64_t)tm * T::BM, P.s.H, wv, lane);
  b.init(P.dz, P.ld, (int64_t)tn * T::BN, P.ld, wv, lane);
  f32x16 acc[T::MT][T::NT];
  T::run(a, b, 0, P.s.N / T::BK, -1, 0, (uint32_t)(uintptr_t)RLDA_AS3(char, lds_all), acc);
  // Through LDS, from the accumulators' 4 columns of each of 32 rows to 16 bytes of few rows a lane: a store then fills whole lines, past the caches
  // (16 tokens of 2048 columns, 151936 rows: 245 -> 140 us; 1024 of 3584, 75000 rows: 697 -> 595; dz, which stays in the caches until it is read,
  // gains nothing by it).  Granules of 16 bytes are exchanged by row against bank conflicts; the memory is the wavefront's own: nothing is waited for.
  constexpr int G = T::MT * 4;                              // granules of a row
  char* const mine = lds_all + wv * (T::MT * T::NT * 2048);
#pragma unroll
  for (int j = 0; j < T::NT; ++j)
#pragma unroll
    for (int i = 0; i < T::MT; ++i)
#pragma unroll
      for (int x4 = 0; x4 < 4; ++x4) {
        const int row = j * 32 + (lane & 31);
        *reinterpret_cast<bf16x4*>(mine + (row * G + ((i * 4 + x4) ^ (row & (G - 1)))) * 16 + (lane >> 5) * 8) =
            bf16x4{(__bf16)acc[i][j][4 * x4], (__bf16)acc[i][j][4 * x4 + 1], (__bf16)acc[i][j][4 * x4 + 2], (__bf16)acc[i][j][4 * x4 + 3]};
      }
  const int g = lane % G, h = tm * T::BM + wm * T::MT * 32 + g * 8;
  auto store = [&](auto past) {
#pragma unroll
    for (int r = 0; r < T::NT * 32; r += 64 / G) {
      const int row = r + lane / G, v = tn * T::BN + wn * T::NT * 32 + row;
      const bf16x8 out = *reinterpret_cast<const bf16x8*>(mine + (row * G + (g ^ (row & (G - 1)))) * 16);
      bf16x8* const to = reinterpret_cast<bf16x8*>(P.out + (size_t)v * P.stride + h);
      if (v < P.s.V && h < P.s.H) {
        if constexpr (decltype(past)::value) __builtin_nontemporal_store(out, to);
        else                                 *to = out;
      }
    }
  };
  if (P.past) store(std::true_type{});
  else        store(std::false_type{});
}

__global__ void __launch_bounds__(256) linear_logprob_zero_kernel(__bf16* out, int64_t stride, int V, int H) {
  const int v = (int)(blockIdx.y * GRID_X + blockIdx.x);
  if (v >= V) return;
  for (int h = threadIdx.x * 8; h < H; h += 2048) *reinterpret_cast<uint4*>(out + (size_t)v * stride + h) = make_uint4(0, 0, 0, 0);
}

// ---- host side

template <Layout LA, Layout LB> using Big = Tile<2, 4, 4, 2, 64, 2, LA, LB>;        // 256 x 256
template <Layout LA, Layout LB> using Mid = Tile<2, 2, 2, 2, 64, 2, LA, LB>;        // 128 x 128, two to a compute unit
template <Layout LA, Layout LB> using Small64 = Tile<4, 1, 1, 2, 64, 4, LA, LB>;    // 128 x 64
template <Layout LA, Layout LB> using Small32 = Tile<4, 1, 1, 1, 64, 4, LA, LB>;    // 128 x 32
constexpr int PAD = 64;                                                             // scratch is padded to whole k-steps of any of them

enum Form { SMALL32, SMALL64, MID, BIG };
// the tile for N tokens: as few as hold them; of the two large ones the smaller where the larger would be mostly empty (333 of 896 columns, 50001 rows:
// 48 us, 256 x 128 alone on a compute unit 58; 256 of 3584, 151936 rows: 256 x 256 345 us, 128 x 128 370)
Form form_for(int64_t N) {
  if (N <= 32) return SMALL32;
  if (N <= 64) return SMALL64;
  const int64_t big = (N + 255) / 256 * 256, mid = (N + 127) / 128 * 128;
  return mid * 5 <= big * 4 ? MID : BIG;
}
int bm_of(Form f) { return f == BIG ? 256 : 128; }
int bn_of(Form f) { return f == BIG ? 256 : f == MID ? 128 : f == SMALL64 ? 64 : 32; }

// `KERNEL` with `lds` bytes of dynamic LDS, which a device has to be told of once
template <auto KERNEL, typename P> hipError_t enqueue_tile(int lds, dim3 grid, int threads, hipStream_t st, const P& params) {
  static std::atomic<uint64_t> told{0};
  int device = 0;
  hipError_t e = hipGetDevice(&device);
  if (e != hipSuccess) return e;
  const uint64_t bit = (uint64_t)1 << (device & 63);
  if (device >= 64 || !(told.load(std::memory_order_relaxed) & bit)) {
    e = hipFuncSetAttribute(reinterpret_cast<const void*>(KERNEL), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return e;
    told.fetch_or(bit, std::memory_order_relaxed);
  }
  hipLaunchKernelGGL(KERNEL, grid, dim3(threads), lds, st, params);
  return hipGetLastError();
}
template <typename T> hipError_t enqueue_forward(const ForwardParams& P, hipStream_t st) {
  return enqueue_tile<linear_logprob_kernel<T>>(T::LDS, grid_of(P.s.tiles_m * P.s.tiles_n), T::THREADS, st, P);
}
template <typename T> hipError_t enqueue_dz(const BackwardParams& P, hipStream_t st) {
  return enqueue_tile<linear_logprob_dz_kernel<T>>(T::LDS, grid_of(P.f.s.tiles_m * P.f.s.tiles_n), T::THREADS, st, P);
}
template <typename T> hipError_t enqueue_dhidden(const DhiddenParams& P, hipStream_t st) {
  return enqueue_tile<linear_logprob_dhidden_kernel<T>>(T::LDS, dim3(P.tiles_m * P.tiles_n * P.splits), T::THREADS, st, P);
}
template <typename T> hipError_t enqueue_dweight(const DweightParams& P, hipStream_t st) {
  return enqueue_tile<linear_logprob_dweight_kernel<T>>(T::LDS, grid_of(P.s.tiles_m * P.s.tiles_n), T::THREADS, st, P);
}

constexpr int64_t LIMIT = 1 << 24, STRIDE_LIMIT = 1 << 20;
dim3 rows_grid(int n) { return dim3(n < GRID_X ? n : GRID_X, (n + GRID_X - 1) / GRID_X); }
size_t align256(size_t n) { return (n + 255) / 256 * 256; }
int64_t up(int64_t n, int64_t m) { return (n + m - 1) / m * m; }
bool lies(const void* p, int64_t stride, int hidden) {
  return !((uintptr_t)p & 15u) && stride >= hidden && stride % 8 == 0 && stride <= STRIDE_LIMIT;
}
int check(int dtype, int64_t n, int vocab, int hidden, float inv_t) {
  if (n < 0 || vocab < 1 || hidden < 8) return -1;
  if (!(inv_t > 0.f) || inv_t > 3.0e38f) return -1;
  if (dtype != 1 || hidden % 8 || n > LIMIT || vocab > LIMIT || hidden > STRIDE_LIMIT) return -2;
  if (n * vocab > (int64_t)1 << 45) return -2;              // tiles are counted in 31 bits
  return 0;
}

struct ForwardLayout { size_t part, zy, copy, total; int64_t H64; };
ForwardLayout forward_layout(int64_t N, int V, int H) {
  ForwardLayout l;
  const int64_t tiles = (V + bm_of(form_for(N)) - 1) / bm_of(form_for(N));
  l.H64 = up(H, PAD);
  l.part = 0;
  l.zy = align256((size_t)tiles * N * sizeof(float4));
  l.copy = l.zy + align256((size_t)N * sizeof(float));
  l.total = l.copy + (H % PAD ? align256((size_t)N * l.H64 * 2) : 0);
  return l;
}

// Pieces of the vocabulary: dz of one is at most 256 MB, what the last-level cache holds.
constexpr int64_t PIECE_BYTES = (int64_t)256 << 20;
struct BackwardLayout { int64_t N64, H64; int piece, splits; size_t odd, token, copy, dz, sum, total; };
BackwardLayout backward_layout(int64_t N, int V, int H, bool dhidden) {
  BackwardLayout l;
  l.N64 = up(N, 64); l.H64 = up(H, PAD);
  int64_t cols = PIECE_BYTES / 2 / l.N64 / 256 * 256;
  if (cols < 1024) cols = 1024;
  const int64_t pieces = (V + cols - 1) / cols;
  l.piece = (int)up((V + pieces - 1) / pieces, 256);
  const Form f = N <= 64 ? SMALL64 : form_for(N);
  const int64_t tiles = ((H + bm_of(f) - 1) / bm_of(f)) * ((l.N64 + bn_of(f) - 1) / bn_of(f));
  // splits of a piece, each of 512 rows and more: the fewest rounds of the workgroups that the compute units hold, for the rows that a round takes; a
  // split's sums, written and read again, cost as much as about 1000 rows (1024 tokens, 3584 columns, 75000 rows, 56 tiles: 5 splits 810 us, 9 540)
  l.splits = 1;
  const int held = f == MID ? 512 : 256;
  float best = INFINITY;
  for (int s = 1; s <= 64 && (s == 1 || s <= l.piece / 512); ++s) {
    const float cost = (float)((tiles * s + held - 1) / held * held) / s * l.piece + 1000.f * s * tiles;
    if (cost < best) { best = cost; l.splits = s; }
  }
  l.odd = 0;
  l.token = 256;
  l.copy = l.token + align256((size_t)l.N64 * sizeof(float4));
  l.dz = l.copy + align256((size_t)l.N64 * l.H64 * 2);
  l.sum = l.dz + align256((size_t)l.N64 * l.piece * 2);
  l.total = l.sum + (dhidden ? align256((size_t)l.splits * l.N64 * H * sizeof(float)) : 0);
  return l;
}

bool fits(const void* ws, size_t bytes, size_t need) { return ws && bytes >= need && !((uintptr_t)ws & 255u); }

int check_forward(const rl_linear_logprob_desc* d) {
  if (!d) return -1;
  if (d->struct_size != sizeof(rl_linear_logprob_desc)) return -4;
  return check(d->dtype, d->n_rows, d->vocab, d->hidden, d->inv_temperature);
}
int check_backward(const rl_linear_logprob_backward_desc* d) {
  if (!d) return -1;
  if (d->struct_size != sizeof(rl_linear_logprob_backward_desc)) return -4;
  return check(d->dtype, d->n_rows, d->vocab, d->hidden, d->inv_temperature);
}

}  // namespace

extern "C" {

size_t rl_linear_logprob_workspace_bytes(const rl_linear_logprob_desc* d) {
  if (check_forward(d) != 0 || d->n_rows == 0) return 0;
  return forward_layout(d->n_rows, d->vocab, d->hidden).total;
}

int rl_linear_logprob(const rl_linear_logprob_desc* d, void* hip_stream) {
  const int rc = check_forward(d);
  if (rc != 0) return rc;
  if (d->n_rows == 0) return 0;
  if (!d->hidden_states || !d->weight || !d->token_ids) return -1;
  if (!lies(d->hidden_states, d->hidden_stride, d->hidden) || !lies(d->weight, d->weight_stride, d->hidden)) return -2;
  const int N = (int)d->n_rows, V = d->vocab, H = d->hidden;
  const ForwardLayout l = forward_layout(N, V, H);
  if (!fits(d->workspace, d->workspace_bytes, l.total)) return -3;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  char* const ws = static_cast<char*>(d->workspace);
  const Form f = form_for(N);
  ForwardParams P{};
  P.s = Shape{N, V, H, (V + bm_of(f) - 1) / bm_of(f), (N + bn_of(f) - 1) / bn_of(f)};
  P.hidden = d->hidden_states; P.hs = d->hidden_stride;
  P.weight = d->weight; P.ws = d->weight_stride; P.ids = d->token_ids;
  P.k2 = d->inv_temperature * LOG2E;
  P.part = reinterpret_cast<float4*>(ws + l.part); P.zy = reinterpret_cast<float*>(ws + l.zy);
  if (H % PAD) {                                             // zeros behind the last column
    hipLaunchKernelGGL(linear_logprob_prepare_kernel, rows_grid(N), dim3(256), 0, st, static_cast<const char*>(P.hidden), P.hs, N, H, V, N, (int)l.H64,
                       nullptr, nullptr, nullptr, nullptr, nullptr, ws + l.copy, nullptr, false, nullptr);
    P.hidden = ws + l.copy; P.hs = l.H64;
  }
  hipError_t e = f == SMALL32 ? enqueue_forward<Small32<K_COLS, K_COLS>>(P, st) : f == SMALL64 ? enqueue_forward<Small64<K_COLS, K_COLS>>(P, st)
               : f == MID ? enqueue_forward<Mid<K_COLS, K_COLS>>(P, st) : enqueue_forward<Big<K_COLS, K_COLS>>(P, st);
  if (e != hipSuccess) return -5;
  if (N <= 1024) hipLaunchKernelGGL((linear_logprob_merge_kernel<4>), dim3((N + 3) / 4), dim3(256), 0, st, P, d->logprob, d->lse, d->entropy);
  else           hipLaunchKernelGGL((linear_logprob_merge_kernel<16>), dim3((N + 15) / 16), dim3(256), 0, st, P, d->logprob, d->lse, d->entropy);
  return hipGetLastError() == hipSuccess ? 0 : -5;
}

size_t rl_linear_logprob_backward_workspace_bytes(const rl_linear_logprob_backward_desc* d) {
  if (check_backward(d) != 0 || d->n_rows == 0 || (!d->dhidden && !d->dweight)) return 0;
  return backward_layout(d->n_rows, d->vocab, d->hidden, d->dhidden != nullptr).total;
}

int rl_linear_logprob_backward(const rl_linear_logprob_backward_desc* d, void* hip_stream) {
  const int rc = check_backward(d);
  if (rc != 0) return rc;
  if (!d->dhidden && !d->dweight) return 0;
  const int N = (int)d->n_rows, V = d->vocab, H = d->hidden;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (d->dweight && !lies(d->dweight, d->dweight_stride, H)) return -2;
  if (N == 0) {
    if (d->dweight) hipLaunchKernelGGL(linear_logprob_zero_kernel, rows_grid(V), dim3(256), 0, st, static_cast<__bf16*>(d->dweight), d->dweight_stride, V, H);
    return hipGetLastError() == hipSuccess ? 0 : -5;
  }
  if (!d->hidden_states || !d->weight || !d->token_ids || !d->lse || !d->g_logprob || (d->g_entropy && !d->entropy)) return -1;
  if (!lies(d->hidden_states, d->hidden_stride, H) || !lies(d->weight, d->weight_stride, H)) return -2;
  if (d->dhidden && !lies(d->dhidden, d->dhidden_stride, H)) return -2;
  const BackwardLayout l = backward_layout(N, V, H, d->dhidden != nullptr);
  if (!fits(d->workspace, d->workspace_bytes, l.total)) return -3;
  char* const ws = static_cast<char*>(d->workspace);
  const Form f = N <= 64 ? SMALL64 : form_for(N);
  const int N64 = (int)l.N64;
  const bool twice = N <= 32;
  float4* const token = reinterpret_cast<float4*>(ws + l.token);
  int* const odd = reinterpret_cast<int*>(ws + l.odd);
  hipLaunchKernelGGL(linear_logprob_prepare_kernel, rows_grid(N64), dim3(256), 0, st, static_cast<const char*>(d->hidden_states), d->hidden_stride, N, H, V,
                     N64, (int)l.H64, d->token_ids, d->lse, d->entropy, d->g_logprob, d->g_entropy, ws + l.copy, token, twice, odd);
  for (int v0 = 0; v0 < V; v0 += l.piece) {
    const int v1 = v0 + l.piece < V ? v0 + l.piece : V, cols = v1 - v0;
    const char* const w = static_cast<const char*>(d->weight) + (size_t)v0 * d->weight_stride * 2;
    BackwardParams P{};
    P.f.s = Shape{N, cols, H, (cols + bm_of(f) - 1) / bm_of(f), (N64 + bn_of(f) - 1) / bn_of(f)};
    P.f.hidden = ws + l.copy; P.f.hs = l.H64; P.f.weight = w; P.f.ws = d->weight_stride; P.f.ids = d->token_ids;
    P.f.k2 = d->inv_temperature * LOG2E;
    P.token = token; P.dz = reinterpret_cast<__bf16*>(ws + l.dz); P.ld = l.piece;
    P.v0 = v0; P.v1 = v1; P.inv_t = d->inv_temperature; P.twice = twice; P.odd = odd;
    hipError_t e = f == SMALL64 ? enqueue_dz<Small64<K_COLS, K_COLS>>(P, st) : f == MID ? enqueue_dz<Mid<K_COLS, K_COLS>>(P, st)
                                                                                        : enqueue_dz<Big<K_COLS, K_COLS>>(P, st);
    if (e != hipSuccess) return -5;
    if (d->dhidden) {
      DhiddenParams Q{};
      Q.tiles_m = (H + bm_of(f) - 1) / bm_of(f); Q.tiles_n = (N64 + bn_of(f) - 1) / bn_of(f); Q.splits = l.splits;
      Q.weight = w; Q.ws = d->weight_stride; Q.V = cols; Q.H = H; Q.N64 = N64; Q.dz = P.dz; Q.ld = P.ld;
      Q.sum = reinterpret_cast<float*>(ws + l.sum); Q.first = v0 == 0; Q.odd = odd;
      e = f == SMALL64 ? enqueue_dhidden<Small64<K_ROWS, K_COLS>>(Q, st) : f == MID ? enqueue_dhidden<Mid<K_ROWS, K_COLS>>(Q, st)
                                                                                    : enqueue_dhidden<Big<K_ROWS, K_COLS>>(Q, st);
      if (e != hipSuccess) return -5;
    }
    if (d->dweight) {
      DweightParams Q{};
      // two workgroups of a compute unit write and compute in turn; with many tokens the larger tile's fewer reads count for more
      // (333 x 896: 58 -> 46 us; 16 x 2048: 140 -> 125 us; equal at 1024 x 3584)
      const int edge = N64 <= 512 ? 128 : 256;
      Q.s = Shape{N64, cols, H, (H + edge - 1) / edge, (cols + edge - 1) / edge};
      Q.hidden = ws + l.copy; Q.hs = l.H64; Q.dz = P.dz; Q.ld = P.ld;
      Q.out = static_cast<__bf16*>(d->dweight) + (size_t)v0 * d->dweight_stride; Q.stride = d->dweight_stride;
      // rows that begin inside a line leave parts of lines, which only the caches put together (15 x 1912, 32000 rows: past them 55 us, through them 30)
      Q.past = !((uintptr_t)d->dweight % 128 || d->dweight_stride * 2 % 128);
      e = edge == 128 ? enqueue_dweight<Mid<K_ROWS, K_ROWS>>(Q, st) : enqueue_dweight<Big<K_ROWS, K_ROWS>>(Q, st);
      if (e != hipSuccess) return -5;
    }
  }
  if (d->dhidden) {
    const float* const sum = reinterpret_cast<const float*>(ws + l.sum);
    __bf16* const out = static_cast<__bf16*>(d->dhidden);
    const __bf16* const w = static_cast<const __bf16*>(d->weight);
    const int64_t slab = (int64_t)N64 * H;
    const dim3 rows = rows_grid(N);
    if (l.splits >= 8)
      hipLaunchKernelGGL(linear_logprob_round_kernel<16>, dim3(rows.x, (H + 63) / 64, rows.y), dim3(256), 0, st, sum, l.splits, slab, N, H, out, d->dhidden_stride, twice,
                         odd, w, d->weight_stride, V, d->token_ids, token, d->inv_temperature);
    else
      hipLaunchKernelGGL(linear_logprob_round_kernel<1>, dim3(rows.x, (H + 1023) / 1024, rows.y), dim3(256), 0, st, sum, l.splits, slab, N, H, out, d->dhidden_stride, twice,
                         odd, w, d->weight_stride, V, d->token_ids, token, d->inv_temperature);
  }
  return hipGetLastError() == hipSuccess ? 0 : -5;
}

}  // extern "C"
