// Causal attention over packed sequences with grouped heads, forward and backward (formulas: include/rl_packed_attn.h).
//
// Matrix-core bound: a key row read from memory meets every row (token, head of the group) of a workgroup.  The rows of a KV head
// are its group's heads of consecutive tokens, so that a block of 128 rows spans few tokens and little work lies above the
// diagonal; blocks are cut from the row of tokens as it is, over the ends of sequences, and every row has its own range of
// keys [start of its sequence, itself].
//
// All products are 32x32x16.  What follows a product (weights, gradients of scores) is done in the registers it leaves, and goes
// into the next product as it lies: a product's rows (m: along the registers) become the next one's contraction index, whose order both
// operands share.  So scores are taken with m = keys forward and for dq (a lane holds one row), with m = rows for dk and dv (a
// lane holds one key); the other operand of the next product is read transposed from LDS in that order.
//   forward   S^T = K Q^T, online softmax (a row's reference moves only when a score passes it by 2^8), O^T += V^T P^T
//   dq        S^T, dP^T = V dO^T, dQ^T += K^T dS^T.  D from the rounded out is off by enough to show in dq and dk beside the rounding of
//             the products' factors (1600 tokens: dq off by 2.57e-3 of its norm, 2.36e-3 with an exact D).  The sum of a row of dS, which would
//             be 0, says by how much: the other kernel gets the exact D, and rows of few keys, where it matters, a second walk over them that
//             adds what is missing, K^T P^T times it, and what the rounding of dS left over (rows of up to 64 keys: 2.29e-3)
//   dk, dv    S = Q K^T, dP = dO V^T, dV^T += dO^T P, dK^T += Q^T dS: a workgroup owns its keys and walks the rows that see them,
//             so heads of a group add up in its registers, in a fixed order, without atomics (the price: S and dP are computed twice).
//             P and dS are rounded for the last two; keys that few rows see also take the products of what that left over
//             (6 sequences of 2 tokens: dk off by 2.55e-3 of its norm, the rounding of the result alone is 1.66e-3)
// Roundings to bf16: P in front of V (out off by 1.9e-3 to 2.1e-3 of its norm), P and dS in the gradients (2.4e-3 in all); two parts of 8 bits each would double a
// product's cost, and are taken where few terms make up a sum.
// Tiles of 64 keys or rows move straight into LDS, two buffers.  Their pattern (xor on a row's 16-byte chunks) lets both the 16-byte reads (16
// rows at one column) and the transposing 8-byte reads (4 rows of 64 bytes) meet no bank conflict.
//
// Measured, 28/4 heads of 128 columns: forward of 8192 tokens 453 us (1.06 Pflop/s), of 10 sequences of 1280 to 1996 240, their dq 350 (0.83 Pflop/s
// over its three products), dk and dv 490 (0.79 over four), at 1.7 GHz with the matrix cores busy 46 to 50 % of the cycles; 14/2 heads of 64, 48 sequences of 24 to 340: 19, 33, 42.
//
// A masked weight is 0, but 0 times infinity is not: whatever a key outside a row's range holds would reach the row through a
// product.  It cannot do so unseen, sums are then not finite; such rows (or keys) are computed again, with zeros in place of what is no number.
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <atomic>
#include <type_traits>

#include "../../include/rl_packed_attn.h"
#include "rlda_tile.h"

namespace {

using namespace rlda;

typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr float LN2 = 0.69314718055994531f, LOG2E = 1.4426950408889634f;
constexpr float LOWEST = -1e30f;                            // a row's reference before its first key
constexpr float SLACK = 8.f;                                // a weight may pass 1 by this power of 2 before the reference follows
constexpr int FEW_KEYS = 64, FEW_ROWS = 64;                 // rows of up to so many keys get a second walk (dq), keys of up to so many rows, too (dk, dv)
constexpr int TILE = 64, WAVES = 4, THREADS = 64 * WAVES, ROWS = 32 * WAVES;

struct Tensor { const char* p; int64_t stride; };           // bytes between tokens
struct Params {
  Tensor q, k, v, dout, out, dq, dk, dv;                    // the last three, and `out` forward, are written
  const int32_t* cu;
  int S, T, Hq, Hkv, r;
  uint32_t magic;                                           // x / r = x * magic >> 16 for x < 1024
  int QB, n_blocks;                                         // tokens a block of rows holds; blocks (of rows or keys)
  float scale, c;                                           // c = |scale| log2 e
  uint32_t flip, keep;                                      // queries get the scale's sign (xor) or are zeros (and)
  float ck, k_down;                                         // c for dk and dv, whose keys are taken times k_down: c, and 1, but for scales next to 0
  float* lse;                                               // [Hq][T]
  int32_t* order;                                           // backward: [k_blocks] blocks of keys in the order in which they are begun, and as many of scratch; or null
  int k_blocks;
  float* stats;                                             // backward: [2][T][Hq]: -lse in units of ck, -D: what the sums of S and dP start from
  int splits;                                               // workgroups that share a block of keys
  float* part;                                              // their sums, if more than one: [splits][2][T][Hkv][d], dk and dv
};

// N steps of products whose fragments are asked for AHEAD steps before; left alone, the compiler asks right before the use, and every product
// waits for LDS.  read(i, fragments), multiply(i, fragments).
template <int N, int AHEAD, typename Read, typename Multiply, int F>
__device__ __forceinline__ void pipeline_steps(Read read, Multiply multiply, bf16x8 (&f)[AHEAD + 1][F]) {
#pragma unroll
  for (int i = 0; i < AHEAD && i < N; ++i) read(i, f[i]);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if (i + AHEAD < N) read(i + AHEAD, f[(i + AHEAD) % (AHEAD + 1)]);
    __builtin_amdgcn_sched_barrier(0);
    multiply(i, f[i % (AHEAD + 1)]);
  }
}
template <typename T> struct FragmentsOf;
template <typename C, int F> struct FragmentsOf<void (C::*)(int, bf16x8 (&)[F]) const> { static constexpr int COUNT = F; };
template <int N, int AHEAD, typename Read, typename Multiply>
__device__ __forceinline__ void pipeline(Read read, Multiply multiply) {
  bf16x8 f[AHEAD + 1][FragmentsOf<decltype(&Read::operator())>::COUNT];
  pipeline_steps<N, AHEAD>(read, multiply, f);
}

__device__ __forceinline__ int uni(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ float half_max(float x) {
  const u32x2 s = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false));
  return fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
}
__device__ __forceinline__ float half_sum(float x) {
  const u32x2 s = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false));
  return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}

// Block and KV head of a workgroup: blocks of a head stay on as few dies as there are for it, whose L2 then holds its keys.
__device__ __forceinline__ bool place(const Params& P, int& blk, int& j) {
  const int b = blockIdx.x;
  if (P.Hkv <= 8 && 8 % P.Hkv == 0) {
    const int g = 8 / P.Hkv, x = b & 7;
    j = x / g;
    blk = (b >> 3) * g + x % g;
  } else {
    j = b % P.Hkv;
    blk = b / P.Hkv;
  }
  return blk < P.n_blocks;
}
// A dimension of a grid holds fewer than 2^32 threads; a launch of more is accepted and runs in part.
bool launches(int64_t grid, int threads) { return grid * threads < (int64_t)1 << 32; }
int64_t grid_of(int64_t n_blocks, int Hkv) {
  if (Hkv <= 8 && 8 % Hkv == 0) return 8 * ((n_blocks + 8 / Hkv - 1) / (8 / Hkv));
  return n_blocks * Hkv;
}

// The sequence of token i: [start, end), or false.  By one lane.
__device__ __forceinline__ bool sequence_of(const Params& P, int i, int& start, int& end) {
  int lo = -1, hi = P.S + 1;                                // cu[lo] <= i < cu[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (P.cu[mid] <= i) lo = mid; else hi = mid;
  }
  if (lo < 0 || lo >= P.S) return false;
  start = min(max(P.cu[lo], 0), i);
  end = max(min(P.cu[lo + 1], P.T), i + 1);
  return true;
}
// The same for a token that all lanes ask for: 64 entries a step.
__device__ __forceinline__ bool sequence_of_all(const Params& P, int i, int& start, int& end) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = P.S + 1;                                  // the entries not known to be <= i (before lo) or > i (from lo + n on)
  while (n > 64) {
    const int step = (n + 63) >> 6, at = lane * step;
    const int c = __popcll(__ballot(at < n && P.cu[lo + min(at, n - 1)] <= i));          // not decreasing: the first c lanes
    if (c == 0) return false;
    lo += (c - 1) * step;
    n = min(step, n - (c - 1) * step);
  }
  const int c = __popcll(__ballot(lane < n && P.cu[lo + min(lane, n - 1)] <= i));
  const int s = uni(lo + c - 1);
  if (s < 0 || s >= P.S) return false;
  start = uni(min(max(P.cu[s], 0), i));
  end = uni(max(min(P.cu[s + 1], P.T), i + 1));
  return true;
}

template <int D> struct Lds {
  static constexpr int ROWB = D * 2, CH = D / 8, RPL = 1024 / ROWB, TILEB = TILE * ROWB, LOADS = TILEB / 1024 / WAVES;
  static constexpr int KS = D / 16, DB = D / 32;            // k-steps over a head's columns; blocks of 32 columns
  __device__ static __forceinline__ int pattern(int row) {
    return D == 128 ? (row & 3) << 2 | ((row >> 2) & 3) : (row & 2) << 1 | ((row >> 2) & 3);
  }
};

// Fragments of tiles in LDS.  `at` is a lane's address in the first tile; a tile's place, its blocks and rows are constants that go into the
// instructions (the loops are unrolled over the two buffers for it), what is left is an xor or nothing.
// The address as one that the compiler knows nothing of: it would keep every variant of it, over 20, in registers of the loop otherwise.
template <typename F> __device__ __forceinline__ F opaque(F f) {
  asm volatile("" : "+v"(f.at));
  return f;
}

// 32 rows at the 16-byte chunk 2 ks + lane / 32, `offset` bytes on; `lds`: a multiple of 256
template <int D> struct RowFragments {
  uint32_t at;
  __device__ __forceinline__ RowFragments(uint32_t lds, int lane) {
    const int row = lane & 31;
    at = lds + row * Lds<D>::ROWB + ((lane >> 5 ^ Lds<D>::pattern(row)) << 4);
  }
  __device__ __forceinline__ bf16x8 get(int offset, int ks) const { return *RLDA_AS3(const bf16x8, (at ^ ks << 5) + offset); }
};
// transposed: 32 columns (block db), 16 rows in the order in which a product leaves them: 4 (lane / 32) + 0..3, and 8 more
template <int D> struct ColFragments {
  uint32_t at;
  __device__ __forceinline__ ColFragments(uint32_t lds, int lane) {
    const int m16 = lane & 15, row = 4 * (lane >> 5) + (m16 >> 2), chunk = 2 * (lane >> 4 & 1) + ((m16 & 3) >> 1);
    at = lds + row * Lds<D>::ROWB + ((chunk ^ Lds<D>::pattern(row)) << 4) + ((m16 & 1) << 3);
  }
  __device__ __forceinline__ bf16x8 get(int offset, int db) const {
    union { s16x4 h[2]; bf16x8 v; } f;
    f.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(RLDA_AS3(s16x4, (at ^ db << 6) + offset));
    f.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(RLDA_AS3(s16x4, (at ^ db << 6 ^ 32) + offset + 8 * Lds<D>::ROWB));
    return f.v;
  }
};
template <int N> using Const = std::integral_constant<int, N>;

__device__ __forceinline__ f32x16 zeros() {
  f32x16 z;
#pragma unroll
  for (int x = 0; x < 16; ++x) z[x] = 0.f;
  return z;
}
__device__ __forceinline__ bf16x8 pack(const f32x16& v, int s) {
  bf16x8 p;
#pragma unroll
  for (int x = 0; x < 8; ++x) p[x] = (__bf16)v[8 * s + x];
  return p;
}
// rows (or keys) of a lane: registers x of a product with m = keys (rows) stand for 8 (x / 4) + 4 (lane / 32) + x % 4 of a block
__device__ __forceinline__ int m_of(int x) { return 8 * (x >> 2) + (x & 3); }

// C^T of 32 columns (registers) of a lane's row, times `f`, to bf16 at `row`: the halves of a pair of lanes exchange 8 bytes, so that each has 16
__device__ __forceinline__ void store_block(char* row, int db, const f32x16& v, float f, int lane, bool ok) {
#pragma unroll
  for (int y = 0; y < 2; ++y) {
    const bf16x4 a = {(__bf16)(v[8 * y] * f), (__bf16)(v[8 * y + 1] * f), (__bf16)(v[8 * y + 2] * f), (__bf16)(v[8 * y + 3] * f)};
    const bf16x4 b = {(__bf16)(v[8 * y + 4] * f), (__bf16)(v[8 * y + 5] * f), (__bf16)(v[8 * y + 6] * f), (__bf16)(v[8 * y + 7] * f)};
    const u32x2 ua = __builtin_bit_cast(u32x2, a), ub = __builtin_bit_cast(u32x2, b);
    const u32x2 s0 = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(ua[0], ub[0], false, false));
    const u32x2 s1 = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(ua[1], ub[1], false, false));
    if (ok) *reinterpret_cast<u32x4*>(row + (32 * db + 16 * y + 8 * (lane >> 5)) * 2) = u32x4{s0[0], s1[0], s0[1], s1[1]};
  }
}
template <int N>
__device__ __forceinline__ bool finite(const f32x16 (&v)[N]) {
  float z = 0.f;
#pragma unroll
  for (int b = 0; b < N; ++b)
#pragma unroll
    for (int x = 0; x < 16; ++x) z = fmaf(v[b][x], 0.f, z);
  return z == 0.f;
}

__device__ __forceinline__ const char* at(const Tensor& t, int token, int head, int rowb) { return t.p + token * t.stride + (int64_t)head * rowb; }
__device__ __forceinline__ char* to(const Tensor& t, int token, int head, int rowb) { return const_cast<char*>(at(t, token, head, rowb)); }

// ---- a block of rows, one to a lane and its partner in the other half
struct Row { int token, head, start; bool ok; };            // keys [start, token]
struct Block {
  int j, t0, lo, hi;                                        // keys [lo, hi) are what any row of the block sees
  int first, last;                                          // this wavefront's tokens
  bool one;                                                 // all rows of the block are of one sequence, which starts at lo
};
__device__ __forceinline__ bool locate(const Params& P, Block& B, Row& R, int wv, int lane) {
  int blk;
  if (!place(P, blk, B.j)) return false;
  blk = P.n_blocks - 1 - blk;                               // those that see the most keys first
  B.t0 = blk * P.QB;
  const int nt = min(P.QB, P.T - B.t0);
  auto token_of = [&](int x) { return (int)((uint32_t)x * P.magic >> 16); };
  const int x = 32 * wv + (lane & 31);
  const int xl = min(x, nt * P.r - 1), tl = token_of(xl);
  R.ok = x < nt * P.r;
  R.token = B.t0 + tl;
  R.head = B.j * P.r + xl - tl * P.r;
  B.first = uni(B.t0 + token_of(min(32 * wv, nt * P.r - 1)));
  B.last = uni(B.t0 + token_of(min(32 * wv + 31, nt * P.r - 1)));
  B.hi = B.t0 + nt;
  B.lo = B.t0;
  int start = 0, end = 0;
  const bool in = sequence_of_all(P, B.t0, start, end);
  if (in) B.lo = start;
  B.one = in && end >= B.hi;
  if (B.one) {
    R.start = start;
  } else if (!sequence_of(P, R.token, R.start, end)) {
    R.start = R.token + 1;
  }
  return true;
}

// loads of a tile of keys [n0, n0 + 64) of head j, of which those from `hi` on do not exist: they read the last one again
template <int D>
__device__ __forceinline__ void issue_keys(const Tensor& t, int j, int n0, int hi, uint32_t lds, int wv, int lane) {
  typedef Lds<D> L;
  const char* const base = t.p + n0 * t.stride + (int64_t)j * L::ROWB;
  const uint32_t stride = (uint32_t)t.stride;
  const int last = hi - 1 - n0;
#pragma unroll
  for (int i = 0; i < L::LOADS; ++i) {
    const int row = (wv * L::LOADS + i) * L::RPL + lane / L::CH, chunk = (lane % L::CH) ^ L::pattern(row);
    load_to_lds(base, (uint32_t)min(row, last) * stride + chunk * 16, lds + (wv * L::LOADS + i) * 1024);
  }
}
template <int D>
__device__ __forceinline__ void load_row(const char* p, int lane, bool ok, uint32_t flip, uint32_t keep, bf16x8 (&f)[Lds<D>::KS]) {
#pragma unroll
  for (int ks = 0; ks < Lds<D>::KS; ++ks) {
    u32x4 v = {0, 0, 0, 0};
    if (ok) v = *reinterpret_cast<const u32x4*>(p + (16 * ks + 8 * (lane >> 5)) * 2);
#pragma unroll
    for (int x = 0; x < 4; ++x) v[x] = (v[x] ^ flip) & keep;
    f[ks] = __builtin_bit_cast(bf16x8, v);
  }
}

// ---- sums that are not finite: rows (or keys) of a wavefront once more, in tiles of 32 of its own LDS, infinities and NaN of the matrices that weights are
// multiplied with read as zeros.  What of them lies in a row's own range is added at the end: how many of a kind, a product of 0 and 1, says whether there
// is one.  Weights go in two parts of 8 bits.  6000 tokens of 7/1 heads of 128 columns, forward and gradient, one token's q, k and v NaN: 0.8 to 1.8 ms, one
// query alone up to 3.6 (0.56 without; one row or key after another 20 to 142).
constexpr int AGAIN = 32;
enum Kind { NOT_A_NUMBER = 1, PLUS_INF = 2, MINUS_INF = 4 };
struct Kinds {                                              // kinds that were met, and the first and last tile that had any (all lanes the same)
  int all, first, last;
  __device__ __forceinline__ Kinds() : all(0), first(INT32_MAX), last(INT32_MIN) {}
  __device__ __forceinline__ void add(int kinds, int tile) {
    const int k = (__any(kinds & 1) ? 1 : 0) | (__any(kinds & 2) ? 2 : 0) | (__any(kinds & 4) ? 4 : 0);
    if (k) { all |= k; first = min(first, tile); last = max(last, tile); }
  }
};

// this wavefront's loads have landed, its LDS operations are done
__device__ __forceinline__ void settled() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory"); }
// What was computed of these before is computed again: it would be kept in registers of the loops in front otherwise.
__device__ __forceinline__ void forget(int& a, int& b, int& c) { asm volatile("" : "+v"(a), "+v"(b), "+v"(c)); }
// a lane or its partner in the other half
__device__ __forceinline__ bool either_half(bool x) {
  const uint64_t m = __ballot(x);
  return (m | m >> 32) >> (threadIdx.x & 31) & 1;
}
// 32 rows from `base` on, of which those past `last` read it again
template <int D>
__device__ __forceinline__ void fetch32(const char* base, int64_t stride, int last, uint32_t lds, int lane) {
  typedef Lds<D> L;
#pragma unroll 1
  for (int i = 0; i < AGAIN / L::RPL; ++i) {
    const int row = i * L::RPL + lane / L::CH, chunk = (lane % L::CH) ^ L::pattern(row);
    load_to_lds(base, (uint32_t)min(row, last) * (uint32_t)stride + chunk * 16, (uint32_t)uni(lds + i * 1024));
  }
}
// the kinds that a tile holds (this lane's part of it), which then has zeros there; ones in the places of kinds `mark` and zeros elsewhere if there is any
template <int D>
__device__ __forceinline__ int tidy32(uint32_t lds, int lane, int mark) {
  int kinds = 0;
#pragma unroll 4
  for (int i = 0; i < AGAIN / Lds<D>::RPL; ++i) {
    const uint32_t a = lds + i * 1024 + lane * 16;
    u32x4 v = *RLDA_AS3(const u32x4, a);
    uint32_t any = 0;                                       // an exponent of ones, of either half of a word
#pragma unroll
    for (int x = 0; x < 4; ++x) any |= (v[x] & 0x7F807F80u) + 0x00800080u;
    if (!(any & 0x80008000u) && !mark) continue;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      uint32_t w = 0;
#pragma unroll
      for (int half = 0; half < 32; half += 16) {
        const uint32_t u = v[x] >> half & 0xFFFFu;
        const int kind = (u & 0x7F80u) != 0x7F80u ? 0 : u & 0x7Fu ? NOT_A_NUMBER : u & 0x8000u ? MINUS_INF : PLUS_INF;
        kinds |= kind;
        w |= (mark ? (kind & mark ? 0x3F80u : 0u) : kind ? 0u : u) << half;
      }
      v[x] = w;
    }
    *RLDA_AS3(u32x4, a) = v;
  }
  settled();
  return kinds;
}
// acc += (columns of the tile) (weights), both halves of 16 rows
template <int D>
__device__ __forceinline__ void add32(f32x16 (&acc)[Lds<D>::DB], const ColFragments<D>& at, const f32x16& w) {
  const ColFragments<D> cols = opaque(at);
#pragma unroll
  for (int y = 0; y < 2; ++y) {
    const bf16x8 p = pack(w, y);
#pragma unroll
    for (int db = 0; db < Lds<D>::DB; ++db) acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(cols.get(y * 16 * Lds<D>::ROWB, db), p, acc[db], 0, 0, 0);
  }
}
__device__ __forceinline__ f32x16 rest_of(const f32x16& w) {
  f32x16 r;
#pragma unroll
  for (int x = 0; x < 16; ++x) r[x] = w[x] - (float)(__bf16)w[x];
  return r;
}

// What is no number among a result's own terms goes into its columns: count(C, kind) says how many there are of a kind, put(db, x, value) replaces register x
// of columns db.  Both infinities make NaN.
template <int D, typename Count, typename Put>
__device__ __forceinline__ void put_kinds(int kinds, Count count, Put put) {
  uint64_t minus = 0;
#pragma unroll 1
  for (int kind = MINUS_INF; kind; kind >>= 1) {
    if (!(kinds & kind)) continue;
    f32x16 C[Lds<D>::DB];
#pragma unroll
    for (int db = 0; db < Lds<D>::DB; ++db) C[db] = zeros();
    count(C, kind);
#pragma unroll
    for (int db = 0; db < Lds<D>::DB; ++db)
#pragma unroll
      for (int x = 0; x < 16; ++x)
        if (C[db][x] > 0.f) {
          const uint64_t bit = (uint64_t)1 << (16 * db + x);
          put(db, x, kind == MINUS_INF ? -INFINITY : kind == PLUS_INF && !(minus & bit) ? INFINITY : NAN);
          if (kind == MINUS_INF) minus |= bit;
        }
  }
}
__device__ __forceinline__ int column_of(int db, int x, int lane) { return 32 * db + m_of(x) + 4 * (lane >> 5); }

// Rows of the forward call; bad_sum: lse as well.  Scores are rounded before a row's largest is taken off, so that rows of scores far beyond 2^31 (whose rounding is more than
// a weight's range) come out too.
template <int D>
__device__ __forceinline__ void rows_again(const Params& P, const Block& B, Row R, bool bad, bool bad_sum, uint32_t lds, int lane) {
  typedef Lds<D> L;
  forget(lane, R.token, R.head);
  constexpr int V = AGAIN * L::ROWB;
  const int h4 = 4 * (lane >> 5);
  const RowFragments<D> lane_rows(lds, lane);
  const ColFragments<D> cols(lds + V, lane);
  auto fetch = [&](const Tensor& t, int n0, uint32_t to) { fetch32<D>(t.p + uni(n0) * t.stride + (int64_t)B.j * L::ROWB, t.stride, B.hi - 1 - n0, to, lane); };
  auto own = [&](int n0, int x) { const int n = n0 + h4 + m_of(x); return n >= R.start && n <= R.token; };
  auto scores = [&](int n0) {
    f32x16 s = zeros();
    bf16x8 qf[L::KS];                                       // read again for every tile, which leaves registers to the sums
    load_row<D>(at(P.q, R.token, R.head, L::ROWB), lane, R.ok, P.flip, P.keep, qf);
    const RowFragments<D> rows = opaque(lane_rows);
#pragma unroll
    for (int ks = 0; ks < L::KS; ++ks) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(rows.get(0, ks), qf[ks], s, 0, 0, 0);
#pragma unroll
    for (int x = 0; x < 16; ++x) s[x] = own(n0, x) ? s[x] * P.c : -INFINITY;
    return s;
  };
  float m = -INFINITY;
  bool none = false;                                        // a score is +inf or NaN: so is all of the row, as it stands
  for (int n0 = B.lo; n0 <= B.last; n0 += AGAIN) {
    settled();
    fetch(P.k, n0, lds);
    settled();
    const f32x16 s = scores(n0);
#pragma unroll
    for (int x = 0; x < 16; ++x) {
      m = fmaxf(m, s[x]);
      none |= !(s[x] < INFINITY);
    }
  }
  m = half_max(m);
  bad &= !either_half(none);
  if (!__any(bad)) return;
  f32x16 O[L::DB];
#pragma unroll
  for (int db = 0; db < L::DB; ++db) O[db] = zeros();
  float l = 0.f;
  Kinds kinds;
#pragma unroll 1
  for (int n0 = B.lo; n0 <= B.last; n0 += AGAIN) {
    settled();
    fetch(P.k, n0, lds);
    fetch(P.v, n0, lds + V);
    settled();
    f32x16 p = scores(n0);
#pragma unroll
    for (int x = 0; x < 16; ++x) {
      p[x] = p[x] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(p[x] - m);
      l += p[x];
    }
    kinds.add(tidy32<D>(lds + V, lane, 0), n0);
    add32<D>(O, cols, p);
    add32<D>(O, cols, rest_of(p));
  }
  l = half_sum(l);
  const float inv = l > 0.f ? 1.f / l : 0.f;                // no live score at all: 0
  char* const out = to(P.out, R.token, R.head, L::ROWB);
#pragma unroll
  for (int db = 0; db < L::DB; ++db) store_block(out, db, O[db], inv, lane, bad);
  if (P.lse && bad && bad_sum && lane < 32) P.lse[(int64_t)R.head * P.T + R.token] = l > 0.f ? (m + __log2f(l)) * LN2 : -INFINITY;
  put_kinds<D>(kinds.all, [&](f32x16 (&C)[L::DB], int kind) {
#pragma unroll 1
    for (int n0 = kinds.first; n0 <= kinds.last; n0 += AGAIN) {
      settled();
      fetch(P.v, n0, lds + V);
      settled();
      tidy32<D>(lds + V, lane, kind);
      f32x16 w;
#pragma unroll
      for (int x = 0; x < 16; ++x) w[x] = own(n0, x) ? 1.f : 0.f;
      add32<D>(C, cols, w);
    }
  }, [&](int db, int x, float value) { if (bad) reinterpret_cast<__bf16*>(out)[column_of(db, x, lane)] = (__bf16)value; });
}

// dq of rows: an infinite or NaN key in a row's own range, whose weight is 0 at best, is NaN
template <int D>
__device__ __forceinline__ void dq_again(const Params& P, const Block& B, Row R, float lse2, float d_exact, bool bad, uint32_t lds, int lane) {
  typedef Lds<D> L;
  forget(lane, R.token, R.head);
  constexpr int V = AGAIN * L::ROWB;
  const int h4 = 4 * (lane >> 5);
  const RowFragments<D> lane_rows(lds, lane);
  const ColFragments<D> cols(lds, lane);
  auto fetch = [&](const Tensor& t, int n0, uint32_t to) { fetch32<D>(t.p + uni(n0) * t.stride + (int64_t)B.j * L::ROWB, t.stride, B.hi - 1 - n0, to, lane); };
  auto own = [&](int n0, int x) { const int n = n0 + h4 + m_of(x); return n >= R.start && n <= R.token; };
  f32x16 A[L::DB];
#pragma unroll
  for (int db = 0; db < L::DB; ++db) A[db] = zeros();
  Kinds kinds;
#pragma unroll 1
  for (int n0 = B.lo; n0 <= B.last; n0 += AGAIN) {
    settled();
    fetch(P.k, n0, lds);
    fetch(P.v, n0, lds + V);
    settled();
    f32x16 s = zeros(), g = zeros();
    bf16x8 qf[L::KS], gf[L::KS];
    load_row<D>(at(P.q, R.token, R.head, L::ROWB), lane, R.ok, P.flip, P.keep, qf);
    load_row<D>(at(P.dout, R.token, R.head, L::ROWB), lane, R.ok, 0u, ~0u, gf);
    const RowFragments<D> rows = opaque(lane_rows);
#pragma unroll
    for (int ks = 0; ks < L::KS; ++ks) {
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(rows.get(0, ks), qf[ks], s, 0, 0, 0);
      g = __builtin_amdgcn_mfma_f32_32x32x16_bf16(rows.get(V, ks), gf[ks], g, 0, 0, 0);
    }
#pragma unroll
    for (int x = 0; x < 16; ++x) g[x] = own(n0, x) ? __builtin_amdgcn_exp2f(fmaf(s[x], P.c, -lse2)) * (g[x] - d_exact) : 0.f;
    settled();
    kinds.add(tidy32<D>(lds, lane, 0), n0);
    add32<D>(A, cols, g);
    add32<D>(A, cols, rest_of(g));
  }
  char* const dq = to(P.dq, R.token, R.head, L::ROWB);
#pragma unroll
  for (int db = 0; db < L::DB; ++db) store_block(dq, db, A[db], P.scale, lane, bad);
  put_kinds<D>(kinds.all ? NOT_A_NUMBER : 0, [&](f32x16 (&C)[L::DB], int) {
#pragma unroll 1
    for (int n0 = kinds.first; n0 <= kinds.last; n0 += AGAIN) {
      settled();
      fetch(P.k, n0, lds);
      settled();
      tidy32<D>(lds, lane, NOT_A_NUMBER | PLUS_INF | MINUS_INF);
      f32x16 w;
#pragma unroll
      for (int x = 0; x < 16; ++x) w[x] = own(n0, x) ? 1.f : 0.f;
      add32<D>(C, cols, w);
    }
  }, [&](int db, int x, float value) { if (bad) reinterpret_cast<__bf16*>(dq)[column_of(db, x, lane)] = (__bf16)value; });
}

// Where there are few blocks of rows, what a call waits for is one block's tiles after one another: TEAMS of four wavefronts then hold the same rows,
// take the tiles in turn and add up at the end.
template <int D, int TEAMS>
__global__ void __launch_bounds__(THREADS * TEAMS, 2) packed_attn_kernel(const Params P) {
  typedef Lds<D> L;
  extern __shared__ __attribute__((aligned(1024))) char lds_all[];
  const int lane = threadIdx.x & 63, wave = uni(threadIdx.x >> 6), wv = wave % WAVES, team = wave / WAVES, h4 = 4 * (lane >> 5);
  Block B;
  Row R;
  if (!locate(P, B, R, wv, lane)) return;
  const uint32_t lds = (uint32_t)(uintptr_t)RLDA_AS3(char, lds_all) + team * 4 * L::TILEB;
  bf16x8 qf[L::KS];
  load_row<D>(at(P.q, R.token, R.head, L::ROWB), lane, R.ok, P.flip, P.keep, qf);
  const RowFragments<D> rows(lds, lane);
  const ColFragments<D> cols(lds, lane);
  f32x16 O[L::DB];
#pragma unroll
  for (int db = 0; db < L::DB; ++db) O[db] = zeros();
  float mc = LOWEST, l = 0.f;                               // reference (base 2), sum of this lane's keys
  const int tiles = (B.hi - B.lo + TILE - 1) / TILE;
  auto issue = [&](int t, int buffer) {
    const uint32_t st = lds + buffer * 2 * L::TILEB;
    issue_keys<D>(P.k, B.j, B.lo + t * TILE, B.hi, st, wv, lane);
    issue_keys<D>(P.v, B.j, B.lo + t * TILE, B.hi, st + L::TILEB, wv, lane);
  };
  auto tile = [&](auto buffer, int t) {
    constexpr int K = decltype(buffer)::value * 2 * L::TILEB, V = K + L::TILEB;
    landed_barrier();
    if (t + TEAMS < tiles) issue(t + TEAMS, 1 - decltype(buffer)::value);
    const int n0 = B.lo + t * TILE;
    if (t >= tiles || n0 > B.last) return;                                // wholly in the future of this wavefront's rows
    f32x16 s[2] = {zeros(), zeros()};
    pipeline<2 * L::KS, 4>([&](int i, bf16x8 (&f)[1]) { f[0] = rows.get(K + (i & 1) * 32 * L::ROWB, i >> 1); },
                           [&](int i, const bf16x8 (&f)[1]) { s[i & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[0], qf[i >> 1], s[i & 1], 0, 0, 0); });
    if (!B.one || n0 + TILE - 1 > B.first) {
      const int a = R.start - n0 - h4, b = R.token - n0 - h4;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int x = 0; x < 16; ++x) {
          const int n = 32 * kb + m_of(x);
          if (n < a || n > b) s[kb][x] = -INFINITY;
        }
    }
    float mx = s[0][0];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int x = 0; x < 16; ++x) mx = fmaxf(mx, s[kb][x]);
    mx = half_max(mx) * P.c;
    if (__any(mx > mc + SLACK)) {
      const float m2 = fmaxf(mc, mx), alpha = __builtin_amdgcn_exp2f(mc - m2);
      l *= alpha;
#pragma unroll
      for (int db = 0; db < L::DB; ++db) O[db] *= alpha;
      mc = m2;
    }
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int x = 0; x < 16; ++x) {
        s[kb][x] = __builtin_amdgcn_exp2f(fmaf(s[kb][x], P.c, -mc));
        l += s[kb][x];
      }
    const bf16x8 p[4] = {pack(s[0], 0), pack(s[0], 1), pack(s[1], 0), pack(s[1], 1)};
    pipeline<4 * L::DB, 4>([&](int i, bf16x8 (&f)[1]) { f[0] = cols.get(V + i / L::DB * 16 * L::ROWB, i % L::DB); },
                           [&](int i, const bf16x8 (&f)[1]) { O[i % L::DB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[0], p[i / L::DB], O[i % L::DB], 0, 0, 0); });
  };
  if (team < tiles) issue(team, 0);
  for (int t = 0; t < tiles; t += 2 * TEAMS) {              // t: team 0's
    tile(Const<0>{}, t + team);
    if (t + TEAMS < tiles) tile(Const<1>{}, t + TEAMS + team);
  }
  l = half_sum(l);
  if constexpr (TEAMS > 1) {
    landed_barrier();                                       // nobody reads the buffers any more
    float* const sums = reinterpret_cast<float*>(lds_all) + wv * (L::DB * 16 + 2) * 64 + lane;
    if (team == 1) {
#pragma unroll
      for (int db = 0; db < L::DB; ++db)
#pragma unroll
        for (int x = 0; x < 16; ++x) sums[(db * 16 + x) * 64] = O[db][x];
      sums[L::DB * 16 * 64] = mc;
      sums[(L::DB * 16 + 1) * 64] = l;
    }
    landed_barrier();
    if (team == 1) return;
    const float m1 = sums[L::DB * 16 * 64], l1 = sums[(L::DB * 16 + 1) * 64];
    const float m2 = fmaxf(mc, m1), a0 = __builtin_amdgcn_exp2f(mc - m2), a1 = __builtin_amdgcn_exp2f(m1 - m2);
    l = l * a0 + l1 * a1;
#pragma unroll
    for (int db = 0; db < L::DB; ++db)
#pragma unroll
      for (int x = 0; x < 16; ++x) O[db][x] = O[db][x] * a0 + sums[(db * 16 + x) * 64] * a1;
    mc = m2;
  }
  const float inv = l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l);          // no key at all: 0
  char* const out = to(P.out, R.token, R.head, L::ROWB);
  float* const lse = P.lse ? P.lse + (int64_t)R.head * P.T + R.token : nullptr;
#pragma unroll
  for (int db = 0; db < L::DB; ++db) store_block(out, db, O[db], inv, lane, R.ok);
  if (lse && R.ok && lane < 32) *lse = l == 0.f ? -INFINITY : (mc + __log2f(l)) * LN2;
  const bool bad_sum = !(l < INFINITY) || (l == 0.f && R.start <= R.token), bad = either_half(R.ok && (bad_sum || !finite(O)));
  landed_barrier();                                         // nobody reads the buffers any more
  if (__any(bad)) rows_again<D>(P, B, R, bad, bad_sum, (uint32_t)(uintptr_t)RLDA_AS3(char, lds_all) + wv * L::TILEB, lane);
}

// Blocks of keys differ in how many rows see them, and with some four of them to a compute unit one that is begun last shows: those of
// many rows come first, in ORDERS classes (not sorted, so that blocks of a sequence, which read the same rows, stay together; 2, 4 and 16 classes were
// within 1 % of 8).  By one wavefront beside the dq blocks, whose time grows with the tokens; and where workgroups are many nothing is gained, and some of
// the reads shared by the heads of a token are lost.  us of the gradient, as they lie / in order (blocks x KV heads): 14/2 heads of 64 columns, 200 to 2000
// tokens a sequence, 22848 tokens 394 / 310, 90821 (1420 x 2) 1205 / 1114, 131079 (2049 x 2) 1678 / 1629, 24 to 340 tokens 22008 141 / 124, 131113 684 / 710;
// 28/4 of 128, 1280 to 1996 tokens, 9351 523 / 448, 16469 (258 x 4) 832 / 821, 25829 (404 x 4) 1276 / 1303, 66530 3252 / 3371; 2/1 of 64, 100 tokens, 22000
// 45 / 42, 131100 (2049 x 1) 158 / 205, 2^20 1290 / 1950.
constexpr int KEY_BLOCK = 64, ORDERS = 8;
bool ordered(int64_t k_blocks, int Hkv, int d) { return k_blocks <= 1536 && k_blocks * Hkv <= (d == 128 ? 1536 : 3072); }
__device__ __forceinline__ void order_key_blocks(const Params& P) {
  const int lane = threadIdx.x & 63, n = P.k_blocks;
  if (threadIdx.x >= 64) return;
  int32_t* const rows = P.order + n;
  int most = 0;
  for (int b0 = 0; b0 < n; b0 += 64) {
    const int b = b0 + lane;
    int r = 0, start, end;
    if (b < n) {
      const int last = min((b + 1) * KEY_BLOCK, P.T) - 1;
      r = (sequence_of(P, last, start, end) ? end : last + 1) - b * KEY_BLOCK;
      rows[b] = r;
    }
    most = max(most, r);
  }
  for (int o = 1; o < 64; o <<= 1) most = max(most, __shfl_xor(most, o, 64));
  const float per = (float)ORDERS / ((float)most + 1.f);
  int at[ORDERS];
#pragma unroll
  for (int c = 0; c < ORDERS; ++c) at[c] = 0;
  auto each = [&](auto use) {
    for (int b0 = 0; b0 < n; b0 += 64) {
      const int b = b0 + lane;
      const int mine = b < n ? min((int)((float)(most - rows[b]) * per), ORDERS - 1) : -1;
#pragma unroll
      for (int c = 0; c < ORDERS; ++c) {
        const uint64_t m = __ballot(mine == c);
        use(c, mine == c, b, __popcll(m & (((uint64_t)1 << lane) - 1)));
        at[c] += __popcll(m);
      }
    }
  };
  each([](int, bool, int, int) {});
  int first = 0;
#pragma unroll
  for (int c = 0; c < ORDERS; ++c) { const int k = at[c]; at[c] = first; first += k; }
  each([&](int c, bool mine, int b, int before) { if (mine) P.order[at[c] + before] = b; });
}

template <int D, int TEAMS>
__global__ void __launch_bounds__(THREADS * TEAMS, 2) packed_attn_dq_kernel(const Params P) {
  typedef Lds<D> L;
  extern __shared__ __attribute__((aligned(1024))) char lds_all[];
  const int lane = threadIdx.x & 63, wave = uni(threadIdx.x >> 6), wv = wave % WAVES, team = wave / WAVES, h4 = 4 * (lane >> 5);
  if (blockIdx.x == gridDim.x - 1) {                        // one workgroup more than there are blocks
    if (P.order) order_key_blocks(P);
    return;
  }
  Block B;
  Row R;
  if (!locate(P, B, R, wv, lane)) return;
  const uint32_t lds = (uint32_t)(uintptr_t)RLDA_AS3(char, lds_all) + team * 4 * L::TILEB;
  auto issue = [&](int t, int buffer) {
    const uint32_t st = lds + buffer * 2 * L::TILEB;
    issue_keys<D>(P.k, B.j, B.lo + t * TILE, B.hi, st, wv, lane);
    issue_keys<D>(P.v, B.j, B.lo + t * TILE, B.hi, st + L::TILEB, wv, lane);
  };
  const int tiles = (B.hi - B.lo + TILE - 1) / TILE;
  if (team < tiles) issue(team, 0);
  bf16x8 qf[L::KS], gf[L::KS];
  load_row<D>(at(P.q, R.token, R.head, L::ROWB), lane, R.ok, P.flip, P.keep, qf);
  load_row<D>(at(P.dout, R.token, R.head, L::ROWB), lane, R.ok, 0u, ~0u, gf);
  float delta = 0.f;
  {
    bf16x8 of[L::KS];
    load_row<D>(at(P.out, R.token, R.head, L::ROWB), lane, R.ok, 0u, ~0u, of);
#pragma unroll
    for (int ks = 0; ks < L::KS; ++ks)
#pragma unroll
      for (int x = 0; x < 8; ++x) delta = fmaf((float)of[ks][x], (float)gf[ks][x], delta);
    delta = half_sum(delta);
  }
  const float lse2 = R.ok ? P.lse[(int64_t)R.head * P.T + R.token] * LOG2E : 0.f;
  const RowFragments<D> lane_rows(lds, lane);
  const ColFragments<D> lane_cols(lds, lane);
  f32x16 A[L::DB];
  float sum = 0.f;                                          // of dS
#pragma unroll
  for (int db = 0; db < L::DB; ++db) A[db] = zeros();
  auto tile = [&](auto buffer, int t) {
    constexpr int K = decltype(buffer)::value * 2 * L::TILEB, V = K + L::TILEB;
    landed_barrier();
    if (t + TEAMS < tiles) issue(t + TEAMS, 1 - decltype(buffer)::value);
    const int n0 = B.lo + t * TILE;
    if (t >= tiles || n0 > B.last) return;
    const bool masked = !B.one || n0 + TILE - 1 > B.first;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      const RowFragments<D> rows = opaque(lane_rows);
      const ColFragments<D> cols = opaque(lane_cols);
      f32x16 s = zeros(), g = zeros();
      pipeline<L::KS, 2>([&](int ks, bf16x8 (&f)[2]) { f[0] = rows.get(K + kb * 32 * L::ROWB, ks); f[1] = rows.get(V + kb * 32 * L::ROWB, ks); },
                         [&](int ks, const bf16x8 (&f)[2]) {
                           s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[0], qf[ks], s, 0, 0, 0);
                           g = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[1], gf[ks], g, 0, 0, 0);
                         });
#pragma unroll
      for (int x = 0; x < 16; ++x) g[x] = __builtin_amdgcn_exp2f(fmaf(s[x], P.c, -lse2)) * (g[x] - delta);
      if (masked) {
        const int a = R.start - n0 - h4, b = R.token - n0 - h4;
#pragma unroll
        for (int x = 0; x < 16; ++x) {
          const int n = 32 * kb + m_of(x);
          if (n < a || n > b) g[x] = 0.f;
        }
      }
#pragma unroll
      for (int x = 0; x < 16; ++x) sum += g[x];
      const bf16x8 d[2] = {pack(g, 0), pack(g, 1)};
      pipeline<2 * L::DB, 4>([&](int i, bf16x8 (&f)[1]) { f[0] = cols.get(K + (2 * kb + i / L::DB) * 16 * L::ROWB, i % L::DB); },
                             [&](int i, const bf16x8 (&f)[1]) { A[i % L::DB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[0], d[i / L::DB], A[i % L::DB], 0, 0, 0); });
    }
  };
  for (int t = 0; t < tiles; t += 2 * TEAMS) {              // t: team 0's
    tile(Const<0>{}, t + team);
    if (t + TEAMS < tiles) tile(Const<1>{}, t + TEAMS + team);
  }
  sum = half_sum(sum);
  if constexpr (TEAMS > 1) {
    landed_barrier();                                       // nobody reads the buffers any more
    float* const sums = reinterpret_cast<float*>(lds_all) + wv * (L::DB * 16 + 1) * 64 + lane;
    if (team == 1) {
#pragma unroll
      for (int db = 0; db < L::DB; ++db)
#pragma unroll
        for (int x = 0; x < 16; ++x) sums[(db * 16 + x) * 64] = A[db][x];
      sums[L::DB * 16 * 64] = sum;
    }
    landed_barrier();
    if (team == 1) return;                                  // barriers from here on are the others'
#pragma unroll
    for (int db = 0; db < L::DB; ++db)
#pragma unroll
      for (int x = 0; x < 16; ++x) A[db][x] += sums[(db * 16 + x) * 64];
    sum += sums[L::DB * 16 * 64];
  }
  if (R.ok && lane < 32) {
    const int64_t i = (int64_t)R.token * P.Hq + R.head;
    P.stats[i] = -lse2 / P.ck;
    P.stats[(int64_t)P.T * P.Hq + i] = -(delta + sum);
  }
  if (!B.one || B.t0 - B.lo < FEW_KEYS) {                   // a row of the block has few keys
    const bool few = R.token - R.start < FEW_KEYS;
    const int from = max(B.lo, B.t0 - FEW_KEYS + 1);
    landed_barrier();                                       // nobody reads the buffers any more
    for (int n0 = from; n0 < B.hi; n0 += TILE) {
      if (n0 != from) landed_barrier();
      issue_keys<D>(P.k, B.j, n0, B.hi, lds, wv, lane);
      issue_keys<D>(P.v, B.j, n0, B.hi, lds + L::TILEB, wv, lane);
      landed_barrier();
      if (n0 > B.last) continue;
      const int a = few ? R.start - n0 - h4 : TILE, b = R.token - n0 - h4;
      const RowFragments<D> rows = opaque(lane_rows);
      const ColFragments<D> cols = opaque(lane_cols);
#pragma unroll 1
      for (int kb = 0; kb < 2; ++kb) {
        f32x16 s = zeros(), g = zeros();
#pragma unroll
        for (int ks = 0; ks < L::KS; ++ks) {                // as in the first walk, to the bit
          s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(rows.get(kb * 32 * L::ROWB, ks), qf[ks], s, 0, 0, 0);
          g = __builtin_amdgcn_mfma_f32_32x32x16_bf16(rows.get(L::TILEB + kb * 32 * L::ROWB, ks), gf[ks], g, 0, 0, 0);
        }
#pragma unroll
        for (int x = 0; x < 16; ++x) {
          const int n = 32 * kb + m_of(x);
          const float p = __builtin_amdgcn_exp2f(fmaf(s[x], P.c, -lse2)), d = p * (g[x] - delta);
          s[x] = n < a || n > b ? 0.f : (d - (float)(__bf16)d) - p * sum;
        }
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const bf16x8 p = pack(s, y);
#pragma unroll
          for (int db = 0; db < L::DB; ++db) A[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(cols.get((2 * kb + y) * 16 * L::ROWB, db), p, A[db], 0, 0, 0);
        }
      }
    }
  }
  char* const dq = to(P.dq, R.token, R.head, L::ROWB);
#pragma unroll
  for (int db = 0; db < L::DB; ++db) store_block(dq, db, A[db], P.scale, lane, R.ok);
  const float d_exact = delta + sum;
  // with lse or D NaN every key's part is NaN, as it stands; a token of no sequence gets 0
  const bool bad = either_half(R.ok && !finite(A) && ((lse2 == lse2 && d_exact == d_exact) || R.start > R.token));
  landed_barrier();                                         // nobody reads the buffers any more
  if (__any(bad)) dq_again<D>(P, B, R, lse2, d_exact, bad, (uint32_t)(uintptr_t)RLDA_AS3(char, lds_all) + wv * L::TILEB, lane);
}

// 64 lanes x 4 bytes
__device__ __forceinline__ void load4_to_lds(const char* base, uint32_t offset, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(lds), "v"(offset), "s"(base));
}

// A workgroup owns 64 keys: 2 wavefronts of 32 each, four times, in groups that take every fourth tile of 32 rows and add up at the end
// (through LDS, in a fixed order).  So few keys to a workgroup because the first keys of a sequence are seen by all of its rows, the last by few.
// All walk the rows from the last one back: workgroups of the same sequence and head then read the same rows at the same time, out of L2.
// K fragments and the sums of dk and dv are in registers; with 128 columns V's fragments no longer fit into the 256 that let
// two wavefronts share a SIMD, and are read from LDS again for every tile.
template <int D> struct Dkdv {
  typedef Lds<D> L;
  static constexpr bool V_IN_LDS = D == 128;
  static constexpr int KEYS = KEY_BLOCK, GROUPS = 4, THREADS = 128 * GROUPS, STEP = 32;
  static constexpr int TILEB = STEP * L::ROWB, LOADS = TILEB / 1024 / 2, STAGE = 2 * TILEB + 512;
  static constexpr int V_BYTES = V_IN_LDS ? KEYS * L::ROWB : 0, SUMS = 2 * L::DB * 16 * 256;            // of a wavefront
  static constexpr int RING = 2 * GROUPS * STAGE, BYTES = V_BYTES + (RING > 4 * SUMS ? RING : 4 * SUMS);
};
// a key's sums: to its row of dk or dv, or to this workgroup's slab of sums where several share the block
template <int D>
__device__ __forceinline__ float* part_of(const Params& P, int key, int j, bool values) {
  const int64_t slab = (int64_t)P.T * P.Hkv * D;
  return P.part + (2 * blockIdx.y + values) * slab + ((int64_t)key * P.Hkv + j) * D;
}
template <int D>
__device__ __forceinline__ void store_key(const Params& P, int key, int j, const f32x16 (&sum)[Lds<D>::DB], bool values, bool these, int lane) {
  typedef Lds<D> L;
  if (P.splits > 1) {
    if (!these) return;
    float* const p = part_of<D>(P, key, j, values) + 4 * (lane >> 5);
#pragma unroll
    for (int db = 0; db < L::DB; ++db)
#pragma unroll
      for (int x4 = 0; x4 < 4; ++x4)
        *reinterpret_cast<float4*>(p + 32 * db + 8 * x4) = make_float4(sum[db][4 * x4], sum[db][4 * x4 + 1], sum[db][4 * x4 + 2], sum[db][4 * x4 + 3]);
    return;
  }
  char* const p = to(values ? P.dv : P.dk, these ? key : 0, j, L::ROWB);
#pragma unroll
  for (int db = 0; db < L::DB; ++db) store_block(p, db, sum[db], values ? 1.f : P.scale, lane, these);
}
// fragments of the keys, one to a lane, as the scores of dk and dv take them
template <int D>
__device__ __forceinline__ void load_keys(const Params& P, int key, int j, bool ok, int lane, bf16x8 (&kf)[Lds<D>::KS]) {
  load_row<D>(at(P.k, key, j, Lds<D>::ROWB), lane, ok, P.flip, P.keep, kf);
  if (P.k_down != 1.f) {
#pragma unroll
    for (int ks = 0; ks < Lds<D>::KS; ++ks)
#pragma unroll
      for (int x = 0; x < 8; ++x) kf[ks][x] = (__bf16)((float)kf[ks][x] * P.k_down);
  }
}

// dk and dv of a wavefront's keys, from the rows that this workgroup's wavefronts had
template <int D>
__device__ __forceinline__ void keys_again(const Params& P, int j, int key, int rlo, int rhi, int n0, int hi, bool bad_k, bool bad_v, uint32_t lds_v, int wv, int lane) {
  typedef Lds<D> L;
  typedef Dkdv<D> M;
  forget(lane, key, rlo);
  const bool ok = key < P.T;
  const int h4 = 4 * (lane >> 5), n_rows = (hi - n0) * P.r, tiles = (n_rows + M::STEP - 1) / M::STEP;
  const RowFragments<D> lane_vrows(lds_v + wv * 32 * L::ROWB, lane);
  // The last rows whose lse or D is NaN: keys that the first sees have NaN in dk and dv, those that the other one sees in dk.  So it stands.
  int no_lse = -1, no_d = -1;
  for (int r0 = n_rows - 1; r0 >= 0 && no_lse < 0; r0 -= 4 * 64) {
    float ls[4], de[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const int rr = max(r0 - 64 * x - lane, 0), tl = rr / P.r;
      const int64_t i = (int64_t)(n0 + tl) * P.Hq + j * P.r + rr - tl * P.r;
      ls[x] = P.stats[i];
      de[x] = P.stats[(int64_t)P.T * P.Hq + i];
    }
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const uint64_t nl = __ballot(ls[x] != ls[x]), nd = __ballot(de[x] != de[x]);
      if (nl && no_lse < 0) no_lse = max(r0 - 64 * x - __builtin_ctzll(nl), 0);
      if (nd && no_d < 0) no_d = max(r0 - 64 * x - __builtin_ctzll(nd), 0);
    }
  }
  bad_k &= !(no_lse >= rlo && no_lse < rhi) && !(no_d >= rlo && no_d < rhi);
  bad_v &= !(no_lse >= rlo && no_lse < rhi);
  if (!__any(bad_k || bad_v)) return;
  // the rows that the wavefronts of this workgroup had, once more, as in the forward call: rows that do not see a key may hold anything
  const uint32_t mine = lds_v + M::V_BYTES + wv * M::STAGE;
  const RowFragments<D> mine_rows(mine, lane);
  auto each = [&](int first_tile, int last_tile, bool bad, auto use) {
#pragma unroll 1
    for (int t = last_tile; t >= first_tile; --t) {
      if ((tiles - 1 - t) / M::GROUPS % P.splits != (int)blockIdx.y || !__any(bad && rlo < (t + 1) * M::STEP && rhi > t * M::STEP)) continue;
      const int first = (uint32_t)(uni(t) * M::STEP) / (uint32_t)P.r, rem = t * M::STEP - first * P.r, tt = n0 + first, last = hi - 1 - tt;
      auto split = [&](int row, int& tl, int& hh) {
        const uint32_t x = rem + row;
        tl = x * P.magic >> 16;
        hh = x - tl * P.r;
        tl = min(tl, last);
      };
      settled();
#pragma unroll 4
      for (int i = 0; i < M::TILEB / 1024; ++i) {
        const int row = i * L::RPL + lane / L::CH, chunk = (lane % L::CH) ^ L::pattern(row);
        int tl, hh;
        split(row, tl, hh);
        const uint32_t in = hh * L::ROWB + chunk * 16;
        load_to_lds(P.q.p + tt * P.q.stride + (int64_t)j * P.r * L::ROWB, tl * (uint32_t)P.q.stride + in, (uint32_t)uni(mine + i * 1024));
        load_to_lds(P.dout.p + tt * P.dout.stride + (int64_t)j * P.r * L::ROWB, tl * (uint32_t)P.dout.stride + in, (uint32_t)uni(mine + M::TILEB + i * 1024));
      }
      int tl, hh;                                           // lse of the 32 rows, and D
      split(lane & 31, tl, hh);
      *RLDA_AS3(float, mine + 2 * M::TILEB + lane * 4) = P.stats[(lane >> 5) * (int64_t)P.T * P.Hq + (int64_t)(tt + tl) * P.Hq + j * P.r + hh];
      settled();
      use(t);
    }
  };
  auto own = [&](int t, int x) { const int rr = t * M::STEP + h4 + m_of(x); return rr >= rlo && rr < rhi; };
  f32x16 dk[L::DB], dv[L::DB];
#pragma unroll
  for (int db = 0; db < L::DB; ++db) { dk[db] = zeros(); dv[db] = zeros(); }
  const ColFragments<D> qcols(mine, lane), gcols(mine + M::TILEB, lane);
  Kinds q_kinds, g_kinds;
  bf16x8 kf[L::KS], vf[M::V_IN_LDS ? 1 : L::KS];
  load_keys<D>(P, ok ? key : 0, j, ok, lane, kf);
  if constexpr (!M::V_IN_LDS) load_row<D>(at(P.v, ok ? key : 0, j, L::ROWB), lane, ok, 0u, ~0u, vf);
  each(0, tiles - 1, bad_k || bad_v, [&](int t) {
    f32x16 s = zeros(), g = zeros();
    const RowFragments<D> rows = opaque(mine_rows), vrows = opaque(lane_vrows);
#pragma unroll
    for (int ks = 0; ks < L::KS; ++ks) {
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(rows.get(0, ks), kf[ks], s, 0, 0, 0);
      bf16x8 v;
      if constexpr (M::V_IN_LDS) v = vrows.get(0, ks);
      else                       v = vf[ks];
      g = __builtin_amdgcn_mfma_f32_32x32x16_bf16(rows.get(M::TILEB, ks), v, g, 0, 0, 0);
    }
#pragma unroll
    for (int x = 0; x < 16; ++x) {
      const uint32_t a = mine + 2 * M::TILEB + (h4 + m_of(x)) * 4;
      s[x] = own(t, x) ? __builtin_amdgcn_exp2f((s[x] + *RLDA_AS3(const float, a)) * P.ck) : 0.f;
      g[x] = own(t, x) ? s[x] * (g[x] + *RLDA_AS3(const float, a + 128)) : 0.f;
    }
    settled();
    q_kinds.add(tidy32<D>(mine, lane, 0), t);
    g_kinds.add(tidy32<D>(mine + M::TILEB, lane, 0), t);
    add32<D>(dv, gcols, s);
    add32<D>(dv, gcols, rest_of(s));
    add32<D>(dk, qcols, g);
    add32<D>(dk, qcols, rest_of(g));
  });
  store_key<D>(P, key, j, dk, false, bad_k, lane);
  store_key<D>(P, key, j, dv, true, bad_v, lane);
#pragma unroll 1
  for (int values = 1; values >= 0; --values) {             // dv, then dk: an infinite or NaN query, whose weight is 0 at best, makes it NaN
    const bool bad = values ? bad_v : bad_k;
    const uint32_t tile = mine + (values ? M::TILEB : 0);
    const ColFragments<D> cols(tile, lane);
    put_kinds<D>(values ? g_kinds.all : q_kinds.all ? NOT_A_NUMBER : 0, [&](f32x16 (&C)[L::DB], int kind) {
      each(values ? g_kinds.first : q_kinds.first, values ? g_kinds.last : q_kinds.last, bad, [&](int t) {
        tidy32<D>(tile, lane, values ? kind : NOT_A_NUMBER | PLUS_INF | MINUS_INF);
        f32x16 w;
#pragma unroll
        for (int x = 0; x < 16; ++x) w[x] = own(t, x) ? 1.f : 0.f;
        add32<D>(C, cols, w);
      });
    }, [&](int db, int x, float value) {
      if (!bad) return;
      const int col = column_of(db, x, lane);
      if (P.splits > 1) part_of<D>(P, key, j, values)[col] = value;
      else              reinterpret_cast<__bf16*>(to(values ? P.dv : P.dk, key, j, L::ROWB))[col] = (__bf16)value;
    });
  }
}

template <int D>
__global__ void __launch_bounds__(Dkdv<D>::THREADS, 2) packed_attn_dkdv_kernel(const Params P) {
  typedef Lds<D> L;
  typedef Dkdv<D> M;
  extern __shared__ __attribute__((aligned(1024))) char lds_all[];
  const int lane = threadIdx.x & 63, wave = uni(threadIdx.x >> 6), wv = wave & 1, group = wave >> 1, h4 = 4 * (lane >> 5);
  int blk, j;
  if (!place(P, blk, j)) return;
  if (P.order) blk = uni(P.order[blk]);
  const int n0 = blk * M::KEYS, nk = min(M::KEYS, P.T - n0), w0 = 32 * wv;
  const uint32_t lds_v = (uint32_t)(uintptr_t)RLDA_AS3(char, lds_all), lds = lds_v + M::V_BYTES + group * 2 * M::STAGE;
  int start, end, hi = n0 + nk;                             // rows of tokens [n0, hi) may see a key of the block
  if (sequence_of_all(P, n0 + nk - 1, start, end)) hi = end;
  const int n_rows = (hi - n0) * P.r, tiles = (n_rows + M::STEP - 1) / M::STEP;
  const char* const s0 = reinterpret_cast<const char*>(P.stats) + (wv == 1 ? (int64_t)P.T * P.Hq * 4 : 0);
  auto issue = [&](int t, int buffer) {                     // this group's tile t
    const uint32_t st = lds + buffer * M::STAGE;
    const int first = (uint32_t)(t * M::STEP) / (uint32_t)P.r, rem = t * M::STEP - first * P.r, tt = n0 + first;
    const char* const qb = P.q.p + tt * P.q.stride + (int64_t)j * P.r * L::ROWB;
    const char* const gb = P.dout.p + tt * P.dout.stride + (int64_t)j * P.r * L::ROWB;
    const int last = hi - 1 - tt;
    uint32_t ln = lane;
    asm volatile("" : "+v"(ln));                            // as above: what follows from the lane stays out of the loop's registers
    auto split = [&](int row, int& tl, int& hh) {           // rows past the last read rows of the last token again
      const uint32_t x = rem + row;
      tl = x * P.magic >> 16;
      hh = x - tl * P.r;
      tl = min(tl, last);
    };
#pragma unroll
    for (int i = 0; i < M::LOADS; ++i) {
      const int row = (wv * M::LOADS + i) * L::RPL + ln / L::CH, chunk = (ln % L::CH) ^ L::pattern(row);
      int tl, hh;
      split(row, tl, hh);
      const uint32_t in = hh * L::ROWB + chunk * 16, dst = st + (wv * M::LOADS + i) * 1024;
      load_to_lds(qb, tl * (uint32_t)P.q.stride + in, dst);
      load_to_lds(gb, tl * (uint32_t)P.dout.stride + in, dst + M::TILEB);
    }
    int tl, hh;                                             // lse or D, 32 lanes' worth (the others repeat)
    split(ln & 31, tl, hh);
    load4_to_lds(s0 + ((int64_t)tt * P.Hq + j * P.r) * 4, (tl * P.Hq + hh) * 4, st + 2 * M::TILEB + wv * 256);
  };
  const int every = M::GROUPS * P.splits;
  int t = tiles - 1 - (int)blockIdx.y * M::GROUPS - group;
  if (t >= 0) issue(t, 0);
  if constexpr (M::V_IN_LDS) {
    if (wave < WAVES) issue_keys<D>(P.v, j, n0, n0 + nk, lds_v, wave, lane);
  }
  // rows [rlo, rhi) from the block's first token on see this lane's key
  const int key = n0 + w0 + (lane & 31);
  const bool ok = key < P.T;
  const int rlo = (key - n0) * P.r;
  int rhi = rlo;
  if (ok && sequence_of(P, key, start, end)) rhi = (end - n0) * P.r;
  const bool whole = w0 + 32 <= nk && __all(rhi == n_rows); // every key of this wavefront is seen by all rows from some row to the last
  bf16x8 kf[L::KS], vf[M::V_IN_LDS ? 1 : L::KS];
  load_row<D>(at(P.k, ok ? key : 0, j, L::ROWB), lane, ok, P.flip, P.keep, kf);
  if constexpr (!M::V_IN_LDS) load_row<D>(at(P.v, ok ? key : 0, j, L::ROWB), lane, ok, 0u, ~0u, vf);
  if (P.k_down != 1.f) {
#pragma unroll
    for (int ks = 0; ks < L::KS; ++ks)
#pragma unroll
      for (int x = 0; x < 8; ++x) kf[ks][x] = (__bf16)((float)kf[ks][x] * P.k_down);
  }
  const int first_row = w0 * P.r, all_past = (w0 + 31) * P.r;
  const RowFragments<D> lane_rows(lds, lane), lane_vrows(lds_v + wv * 32 * L::ROWB, lane);
  const ColFragments<D> lane_cols(lds, lane);
  f32x16 dk[L::DB], dv[L::DB];
#pragma unroll
  for (int db = 0; db < L::DB; ++db) { dk[db] = zeros(); dv[db] = zeros(); }
  const int rounds = (tiles + every - 1) / every;
  const bool few = rounds == 1 || rhi - rlo <= FEW_ROWS, fine = __any(few && rhi > rlo);
  auto tile = [&](auto buffer, auto rest) {                 // rest: what the rounding of P and dS left over
    constexpr int Q = decltype(buffer)::value * M::STAGE, G = Q + M::TILEB, STATS = G + M::TILEB;
    constexpr bool REST = decltype(rest)::value;
    if constexpr (!REST) {
      landed_barrier();
      if (t >= every) issue(t - every, 1 - decltype(buffer)::value);
    }
    if (t < 0 || (t + 1) * M::STEP <= first_row || w0 >= nk) return;                       // none, or all before this wavefront's first key
    if constexpr (REST) {
      if (!__any(few && rlo < (t + 1) * M::STEP && rhi > t * M::STEP)) return;              // no row of such a key
    }
    const RowFragments<D> rows = opaque(lane_rows), vrows = opaque(lane_vrows);
    const ColFragments<D> cols = opaque(lane_cols);
    typedef float f32x4 __attribute__((ext_vector_type(4)));
    f32x16 s, g;                                            // from -lse / c and -D on
#pragma unroll
    for (int x4 = 0; x4 < 4; ++x4) {
      const uint32_t a = lds + h4 * 4 + STATS + 32 * x4;
      const f32x4 ls = *RLDA_AS3(const f32x4, a), de = *RLDA_AS3(const f32x4, a + 256);
#pragma unroll
      for (int x = 0; x < 4; ++x) { s[4 * x4 + x] = ls[x]; g[4 * x4 + x] = de[x]; }
    }
    __builtin_amdgcn_s_setprio(1);                          // products before the other wavefront's arithmetic: 10 sequences of up to 1996 tokens of 28/4 heads 620 -> 585 us
    pipeline<L::KS, 2>([&](int ks, bf16x8 (&f)[3]) {
      f[0] = rows.get(Q, ks);
      f[1] = rows.get(G, ks);
      if constexpr (M::V_IN_LDS) f[2] = vrows.get(0, ks);
      else                       f[2] = vf[ks];
    }, [&](int ks, const bf16x8 (&f)[3]) {
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[0], kf[ks], s, 0, 0, 0);
      g = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[1], f[2], g, 0, 0, 0);
    });
    __builtin_amdgcn_s_setprio(0);
#pragma unroll
    for (int x = 0; x < 16; ++x) {
      s[x] = __builtin_amdgcn_exp2f(s[x] * P.ck);
      g[x] *= s[x];
    }
    if (!whole || t * M::STEP < all_past || (t + 1) * M::STEP > n_rows) {
      const int a = rlo - t * M::STEP - h4, b = rhi - t * M::STEP - h4;
#pragma unroll
      for (int x = 0; x < 16; ++x)
        if (m_of(x) < a || m_of(x) >= b) { s[x] = 0.f; g[x] = 0.f; }
    }
    if constexpr (REST) {
#pragma unroll
      for (int x = 0; x < 16; ++x) {
        s[x] = few ? s[x] - (float)(__bf16)s[x] : 0.f;
        g[x] = few ? g[x] - (float)(__bf16)g[x] : 0.f;
      }
    }
    bf16x8 p[2] = {pack(s, 0), pack(s, 1)}, d[2] = {pack(g, 0), pack(g, 1)};
    __builtin_amdgcn_s_setprio(1);
    pipeline<2 * L::DB, 2>([&](int i, bf16x8 (&f)[2]) {
      f[0] = cols.get(G + i / L::DB * 16 * L::ROWB, i % L::DB);
      f[1] = cols.get(Q + i / L::DB * 16 * L::ROWB, i % L::DB);
    }, [&](int i, const bf16x8 (&f)[2]) {
      dv[i % L::DB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[0], p[i / L::DB], dv[i % L::DB], 0, 0, 0);
      dk[i % L::DB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[1], d[i / L::DB], dk[i % L::DB], 0, 0, 0);
    });
    __builtin_amdgcn_s_setprio(0);
  };
  for (int round = 0; round < rounds; round += 2) {
    tile(Const<0>{}, Const<0>{});
    if (fine) tile(Const<0>{}, Const<1>{});                 // once more, from the same buffer
    t -= every;
    if (round + 1 < rounds) {
      tile(Const<1>{}, Const<0>{});
      if (fine) tile(Const<1>{}, Const<1>{});
    }
    t -= every;
  }
  // groups 2 and 3 leave their sums for 0 and 1, then 1 for 0
  float* const sums = reinterpret_cast<float*>(lds_all + M::V_BYTES) + lane;
#pragma unroll
  for (int half = M::GROUPS / 2; half >= 1; half >>= 1) {
    landed_barrier();
    float* const mine = sums + (group % half * 2 + wv) * (M::SUMS / 4);
    if (group >= half && group < 2 * half) {
#pragma unroll
      for (int db = 0; db < L::DB; ++db)
#pragma unroll
        for (int x = 0; x < 16; ++x) {
          mine[(db * 16 + x) * 64] = dk[db][x];
          mine[((L::DB + db) * 16 + x) * 64] = dv[db][x];
        }
    }
    landed_barrier();
    if (group < half) {
#pragma unroll
      for (int db = 0; db < L::DB; ++db)
#pragma unroll
        for (int x = 0; x < 16; ++x) {
          dk[db][x] += mine[(db * 16 + x) * 64];
          dv[db][x] += mine[((L::DB + db) * 16 + x) * 64];
        }
    }
  }
  if (group > 0) return;
  store_key<D>(P, key, j, dk, false, ok, lane);
  store_key<D>(P, key, j, dv, true, ok, lane);
  const bool bad_k = either_half(ok && !finite(dk)), bad_v = either_half(ok && !finite(dv));
  landed_barrier();                                         // the other wavefront has read its sums
  if (__any(bad_k || bad_v)) keys_again<D>(P, j, key, rlo, rhi, n0, hi, bad_k, bad_v, lds_v, wv, lane);
}

// The sums of the workgroups that share a block of keys, in their order: a wavefront to a key and head.
template <int D>
__global__ void __launch_bounds__(256) packed_attn_join_kernel(const Params P) {
  typedef Lds<D> L;
  const int lane = threadIdx.x & 63, i = uni(blockIdx.x * 4 + (threadIdx.x >> 6));
  if (i >= P.T * P.Hkv) return;
  const int n = i / P.Hkv, j = i - n * P.Hkv;
  const int64_t slab = (int64_t)P.T * P.Hkv * D;
  constexpr int N = D / 64;
  float k[N] = {}, v[N] = {};
  for (int s = 0; s < P.splits; ++s) {
    const float* const p = P.part + 2 * s * slab + (int64_t)i * D + lane * N;
#pragma unroll
    for (int x = 0; x < N; ++x) { k[x] += p[x]; v[x] += p[slab + x]; }
  }
  __bf16* const pk = reinterpret_cast<__bf16*>(to(P.dk, n, j, L::ROWB)) + lane * N;
  __bf16* const pv = reinterpret_cast<__bf16*>(to(P.dv, n, j, L::ROWB)) + lane * N;
#pragma unroll
  for (int x = 0; x < N; ++x) { pk[x] = (__bf16)(k[x] * P.scale); pv[x] = (__bf16)v[x]; }
}

// ---- host side
template <auto KERNEL> hipError_t enqueue(int lds, int64_t grid, hipStream_t st, const Params& P, int threads = THREADS, int grid_y = 1) {
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
  hipLaunchKernelGGL(KERNEL, dim3((unsigned)grid, grid_y), dim3(threads), lds, st, P);
  return hipGetLastError();
}

constexpr float MOST_SCALE = 2e38f;                         // times log2 e it is still a number
// Sums of S start from -lse / c in dk, dv.  Scales below this would take that past the largest number; keys are then taken times 2^-64 and c times 2^64.
// Whatever that loses of a key (below 2^-62) is times a query (below 2^128) and c still far below a weight's own rounding.
constexpr float LEAST_C = 0x1p-100f;

int check(int dtype, int64_t T, int S, int Hq, int Hkv, int d, float scale) {
  if (T < 0 || S < 0 || Hq <= 0 || Hkv <= 0 || d <= 0) return -1;
  if (!(scale >= -MOST_SCALE && scale <= MOST_SCALE)) return -1;
  if (dtype != 1 || (d != 64 && d != 128) || Hq % Hkv || Hq / Hkv > 64 || Hq > (1 << 16)) return -2;
  if (T > (1 << 24) || S > (1 << 30) || T * Hq > (int64_t)1 << 36) return -2;
  return 0;
}
bool lies(const void* p, int64_t stride, int H, int d, int64_t T) {
  if ((uintptr_t)p & 15u) return false;
  if (stride % 8 || stride < 0 || stride > ((int64_t)1 << 23)) return false;
  return T <= 1 || stride >= (int64_t)H * d;
}
template <typename Desc> void common(Params& P, const Desc* d) {
  P.q = Tensor{static_cast<const char*>(d->q), d->q_stride * 2};
  P.k = Tensor{static_cast<const char*>(d->k), d->k_stride * 2};
  P.v = Tensor{static_cast<const char*>(d->v), d->v_stride * 2};
  P.out = Tensor{static_cast<const char*>(d->out), d->out_stride * 2};
  P.cu = d->cu_seqlens; P.S = d->n_seqs; P.T = (int)d->T;
  P.Hq = d->Hq; P.Hkv = d->Hkv; P.r = d->Hq / d->Hkv;
  P.magic = (65536u + P.r - 1) / P.r;
  P.QB = ROWS / P.r; P.n_blocks = (P.T + P.QB - 1) / P.QB;
  P.scale = d->scale;
  const float m = d->scale < 0.f ? -d->scale : d->scale;
  P.c = m > 0.f ? m * LOG2E : 1.f;
  const bool down = P.c < LEAST_C;
  P.ck = down ? P.c * 0x1p64f : P.c; P.k_down = down ? 0x1p-64f : 1.f;
  P.flip = d->scale < 0.f ? 0x80008000u : 0u; P.keep = m > 0.f ? ~0u : 0u;
}
int check_backward(const rl_packed_attn_backward_desc* d) {
  if (!d) return -1;
  if (d->struct_size != sizeof(rl_packed_attn_backward_desc)) return -4;
  return check(d->dtype, d->T, d->n_seqs, d->Hq, d->Hkv, d->d, d->scale);
}
int64_t key_blocks(int64_t T) { return (T + KEY_BLOCK - 1) / KEY_BLOCK; }
// Workgroups to a block of keys, each of 512 rows and more: as many as find places at once where blocks are few (us without / with: 8 sequences of 64 to 452 tokens of
// 16/2 heads of 128 columns 71 / 38, 1100 of 28/4 109 / 53, 4 x 1024 of 14/2 of 64 columns 68 / 46); two where blocks of long sequences are some 1.5 to a compute
// unit.  What two have to gain there is half of the longest block's time, what they cost is their sums, written and read again: so many rows for each block, fewer
// where there are several sequences, whose lengths may differ (gradient of so many blocks and mean rows a sequence of 128 columns, one / two.  One sequence: 264,
// 4224 152 / 161, 264, 8448 272 / 258, 392, 6272 216 / 236, 392, 43904 1029 / 989.  Two to five: 264, 2112 103 / 111, 392, 2508 136 / 156, 392, 4181 187 / 201, 330, 5280
// 215 / 206, 392, 8780 313 / 290.  Eight and more, lengths alike: 264, 2464 101 / 113, 392, 3658 142 / 171, 264, 5913 181 / 167; up to twice the mean: 264, 2464 155 / 132,
// 392, 3658 228 / 207.  64 columns lie alike.  Above: 460, 17173 524 / 529 and 559 / 539.)
int splits_for(int64_t T, int S, int Hq, int Hkv) {
  const int64_t blocks = key_blocks(T) * Hkv, rows = T * (Hq / Hkv) / (S > 0 ? S : 1);
  int64_t s = 256 / blocks;
  const int64_t least = S <= 1 ? 32 * blocks : S < 8 ? 10 * blocks : 2048;
  if (s < 2 && blocks < 400 && rows >= least) s = 2;
  if (s > rows / 512) s = rows / 512;
  return (int)(s < 1 ? 1 : s > 8 ? 8 : s);
}
struct BackwardLayout { size_t order, part, total; int splits; };
BackwardLayout layout_for(const rl_packed_attn_backward_desc* d) {
  BackwardLayout l;
  l.splits = splits_for(d->T, d->n_seqs, d->Hq, d->Hkv);
  l.order = (size_t)d->T * d->Hq * 2 * sizeof(float);
  l.part = (l.order + (size_t)key_blocks(d->T) * 2 * sizeof(int32_t) + 255) & ~(size_t)255;
  l.total = l.splits > 1 ? l.part + (size_t)l.splits * 2 * d->T * d->Hkv * d->d * sizeof(float) : l.order + (size_t)key_blocks(d->T) * 2 * sizeof(int32_t);
  return l;
}

// Two teams where the blocks find places at once and the tiles of a block are many: for 128 columns, two teams of which fill a compute unit, from 768 tokens
// a sequence on, for 64 from 256 (us, forward and dq, one team / two: 3 x 1000 to 1500 of 8/2 heads of 128 columns 44 + 62 / 34 + 50, 2 x 1000 of 16/16 32 + 49 / 26 + 43,
// 4000 of 16/2 90 + 124 / 81 + 118, 6 x 512 of 16/2 24 + 32 / 26 + 39; 2 x 512 of 14/2 of 64 columns 14.9 + 23.4 / 12.5 + 20.4, 4 x 1024 30 + 41 / 26 + 41).
bool two_teams(const Params& P, int d) {
  return (int64_t)P.n_blocks * P.Hkv <= 512 && P.T >= (int64_t)(d == 128 ? 768 : 256) * P.S;
}
template <int D> hipError_t enqueue_forward(const Params& P, hipStream_t st) {
  constexpr int LDS = 4 * Lds<D>::TILEB;
  const int64_t grid = grid_of(P.n_blocks, P.Hkv);
  return two_teams(P, D) ? enqueue<packed_attn_kernel<D, 2>>(2 * LDS, grid, st, P, 2 * THREADS) : enqueue<packed_attn_kernel<D, 1>>(LDS, grid, st, P);
}
template <int D> hipError_t enqueue_backward(Params& P, hipStream_t st) {
  constexpr int LDS = 4 * Lds<D>::TILEB;
  P.k_blocks = (int)key_blocks(P.T);
  const int64_t grid = grid_of(P.n_blocks, P.Hkv) + 1;
  hipError_t e = two_teams(P, D) ? enqueue<packed_attn_dq_kernel<D, 2>>(2 * LDS, grid, st, P, 2 * THREADS)
                                                        : enqueue<packed_attn_dq_kernel<D, 1>>(LDS, grid, st, P);
  if (e != hipSuccess) return e;
  P.n_blocks = P.k_blocks;
  e = enqueue<packed_attn_dkdv_kernel<D>>(Dkdv<D>::BYTES, grid_of(P.n_blocks, P.Hkv), st, P, Dkdv<D>::THREADS, P.splits);
  if (e != hipSuccess || P.splits == 1) return e;
  return enqueue<packed_attn_join_kernel<D>>(0, ((int64_t)P.T * P.Hkv + 3) / 4, st, P);
}

}  // namespace

extern "C" {

int rl_packed_attn(const rl_packed_attn_desc* d, void* hip_stream) {
  if (!d) return -1;
  if (d->struct_size != sizeof(rl_packed_attn_desc)) return -4;
  const int rc = check(d->dtype, d->T, d->n_seqs, d->Hq, d->Hkv, d->d, d->scale);
  if (rc != 0) return rc;
  if (d->T == 0) return 0;
  if (!d->q || !d->k || !d->v || !d->cu_seqlens || !d->out) return -1;
  if (!lies(d->q, d->q_stride, d->Hq, d->d, d->T) || !lies(d->k, d->k_stride, d->Hkv, d->d, d->T) || !lies(d->v, d->v_stride, d->Hkv, d->d, d->T) ||
      !lies(d->out, d->out_stride, d->Hq, d->d, d->T)) return -2;
  Params P{};
  common(P, d);
  P.lse = d->lse;
  if (!launches(grid_of(P.n_blocks, P.Hkv), THREADS)) return -2;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  const hipError_t e = d->d == 128 ? enqueue_forward<128>(P, st) : enqueue_forward<64>(P, st);
  return e == hipSuccess ? 0 : -5;
}

size_t rl_packed_attn_backward_workspace_bytes(const rl_packed_attn_backward_desc* d) { return check_backward(d) == 0 && d->T > 0 ? layout_for(d).total : 0; }

int rl_packed_attn_backward(const rl_packed_attn_backward_desc* d, void* hip_stream) {
  const int rc = check_backward(d);
  if (rc != 0) return rc;
  if (d->T == 0) return 0;
  if (!d->dout || !d->q || !d->k || !d->v || !d->out || !d->lse || !d->cu_seqlens || !d->dq || !d->dk || !d->dv) return -1;
  if (!lies(d->dout, d->dout_stride, d->Hq, d->d, d->T) || !lies(d->q, d->q_stride, d->Hq, d->d, d->T) || !lies(d->k, d->k_stride, d->Hkv, d->d, d->T) ||
      !lies(d->v, d->v_stride, d->Hkv, d->d, d->T) || !lies(d->out, d->out_stride, d->Hq, d->d, d->T) || !lies(d->dq, d->dq_stride, d->Hq, d->d, d->T) ||
      !lies(d->dk, d->dk_stride, d->Hkv, d->d, d->T) || !lies(d->dv, d->dv_stride, d->Hkv, d->d, d->T)) return -2;
  Params P{};
  common(P, d);
  if (!launches(grid_of(P.n_blocks, P.Hkv) + 1, THREADS) || !launches(grid_of(key_blocks(P.T), P.Hkv), Dkdv<128>::THREADS)) return -2;
  const BackwardLayout l = layout_for(d);
  if (!d->workspace || d->workspace_bytes < l.total || ((uintptr_t)d->workspace & 255u)) return -3;
  P.dout = Tensor{static_cast<const char*>(d->dout), d->dout_stride * 2};
  P.dq = Tensor{static_cast<const char*>(d->dq), d->dq_stride * 2};
  P.dk = Tensor{static_cast<const char*>(d->dk), d->dk_stride * 2};
  P.dv = Tensor{static_cast<const char*>(d->dv), d->dv_stride * 2};
  P.lse = const_cast<float*>(d->lse);
  char* const ws = static_cast<char*>(d->workspace);
  P.stats = reinterpret_cast<float*>(ws);
  P.order = ordered(key_blocks(P.T), P.Hkv, d->d) ? reinterpret_cast<int32_t*>(ws + l.order) : nullptr;
  P.part = reinterpret_cast<float*>(ws + l.part);
  P.splits = l.splits;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  return (d->d == 128 ? enqueue_backward<128>(P, st) : enqueue_backward<64>(P, st)) == hipSuccess ? 0 : -5;
}

}  // extern "C"
