// Norms of queries and keys per head and the rotary embedding over packed tokens, forward and backward
// (formulas: include/rl_qk_norm_rope.h).
//
// Element-wise but for one sum over a head, so HBM bounds it: every head is read once and written once, 16 bytes a lane.  A
// lane holds N elements of a head's lower half and the N they are rotated with (16 bytes each), so D / (2 N) neighbouring lanes
// hold a head, add up its squares by lane exchanges, and need nothing else from each other.  The D / 2 angles of a token are
// shared by its heads: a workgroup takes TB tokens, evaluates their angles once (in turns, reduced to a fraction in fp64: an
// fp32 product of position and frequency would be off by 2e-3 rad at position 32k) and keeps cosines and sines in LDS.
// The next head's loads are issued before the present one's arithmetic.  Stores go past the caches, and so do loads of calls
// that read more than the last-level cache holds (smaller ones may find there what a projection has just left).  us, inputs
// changing, all through the caches / stores past them / loads too / by this rule: 40960 tokens of 28/4 heads of 128 bf16 forward
// 126.6 / 123.5 / 119.9 / 119.9 (5.6 TB/s), 16384 forward and backward 139.6 / 122.9 / 131.3 / 121.0.  A consumer finds less in the caches then: the forward call and
// attention over its outputs, in a graph, stores through / past the caches 9.9 / 10.4 (64 tokens of 28/4 heads of 128), 45.2 / 47.5 (4096), 142 / 146 (16384), 14.9 / 15.1
// (2048 of 14/2 of 64), 29.4 / 29.1 (8192), the forward call alone 14.7 / 12.3 (4096 of 28/4).
//
// Backward, a lane also sums g x rs of its elements over all heads it meets; lanes, wavefronts and then workgroups are added
// in a fixed order (the last by a second kernel, in fp64).
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/rl_qk_norm_rope.h"

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int NT = 256;
constexpr int MAX_GROUPS = 1024;                            // workgroups of a backward call: rows of its workspace
constexpr int GRID_X = 1 << 22;                             // workgroups along x of a forward call: a dimension of a grid holds fewer than 2^32 threads, and one of more runs in part

struct Side {                                               // queries or keys
  const char* x; const char* dy; char* out;                 // dy: backward only
  const float* w; int H;
  int64_t xs, dys, outs;                                    // bytes between tokens
};
// What a lane needs of its row's side.  The fields are read from the arguments before, once: picked by address they are loaded
// again, by every lane, in front of every row's own loads, which then wait for them.
struct Pick {
  const char* x; const char* dy; char* out; int64_t xs, dys, outs; bool norm;
};
struct Params {
  Side q, k;
  const int32_t* pos; const float* inv_freq;
  int T, s0, s1;
  float eps;
  float* part;                                              // backward: [groups][2][D]
};

template <typename T> struct Vec;                           // 16 bytes
template <> struct Vec<float> {
  static constexpr int N = 4;
  __device__ static void get(const u32x4& c, float (&f)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(c[i]);
  }
  __device__ static u32x4 put(const float (&f)[4]) {
    return u32x4{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
  }
};
template <> struct Vec<__bf16> {
  static constexpr int N = 8;
  __device__ static void get(const u32x4& c, float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(c[i] << 16);
      f[2 * i + 1] = __uint_as_float(c[i] & 0xFFFF0000u);
    }
  }
  __device__ static u32x4 put(const float (&f)[8]) {        // nearest even, NaN stays NaN
    typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
    bf16x8 v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (__bf16)f[i];
    return __builtin_bit_cast(u32x4, v);
  }
};

template <bool PAST> __device__ __forceinline__ u32x4 load16(const char* p) {
  if constexpr (PAST) return __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
  return *reinterpret_cast<const u32x4*>(p);
}
__device__ __forceinline__ void store16(char* p, const u32x4& v) { __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(p)); }

template <int D, int TB>
struct Shared {
  __attribute__((aligned(16))) float cs[TB][D / 2], sn[TB][D / 2], w[2][D];
};

template <int D, int TB>
__device__ __forceinline__ void load_weights(const Params& P, Shared<D, TB>& S) {
  const int i = threadIdx.x & (D - 1), side = threadIdx.x / D;
  const float* const w = side ? P.k.w : P.q.w;
  if (side < 2 && w) S.w[side][i] = w[i];
}
template <int D, int TB>
__device__ __forceinline__ void load_angles(const Params& P, Shared<D, TB>& S, int t0, int nt) {
  for (int x = threadIdx.x; x < nt * (D / 2); x += NT) {
    const int tl = x / (D / 2), i = x & (D / 2 - 1);
    const int axis = i < P.s0 ? 0 : (i < P.s0 + P.s1 ? 1 : 2);
    const double turns = (double)P.pos[(size_t)axis * P.T + t0 + tl] * (double)P.inv_freq[i] * 0.15915494309189533577;
    float s, c;
    sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
    S.cs[tl][i] = c; S.sn[tl][i] = s;
  }
}
template <int N>
__device__ __forceinline__ void lds_get(const float* p, float (&f)[N]) {
#pragma unroll
  for (int i = 0; i < N; i += 4) {
    const float4 v = *reinterpret_cast<const float4*>(p + i);
    f[i] = v.x; f[i + 1] = v.y; f[i + 2] = v.z; f[i + 3] = v.w;
  }
}
template <int LANES>
__device__ __forceinline__ float head_sum(float v) {
#pragma unroll
  for (int o = 1; o < LANES; o <<= 1) v += __shfl_xor(v, o, 64);
  return v;
}

__device__ __forceinline__ Pick pick(bool keys, const Side& q, const Side& k) {
  return Pick{keys ? k.x : q.x, keys ? k.dy : q.dy, keys ? k.out : q.out, keys ? k.xs : q.xs, keys ? k.dys : q.dys, keys ? k.outs : q.outs,
              keys ? k.w != nullptr : q.w != nullptr};
}

// the rows (token, head) of a block that a thread's group of lanes takes: every ROWS-th
struct Row {
  int tl, h;
  __device__ __forceinline__ void next(int rows, int H) {
    h += rows;
    while (h >= H) { h -= H; ++tl; }
  }
};

template <typename T, int D, int TB, bool PAST>
__global__ void __launch_bounds__(NT) qk_norm_rope_kernel(const Params P) {
  constexpr int N = Vec<T>::N, LANES = D / 2 / N, ROWS = NT / LANES;
  __shared__ Shared<D, TB> S;
  const int blk = (int)(blockIdx.y * GRID_X + blockIdx.x);
  if (blk >= (P.T + TB - 1) / TB) return;
  const int t0 = blk * TB, nt = min(TB, P.T - t0), H = P.q.H + P.k.H;
  const int i0 = (threadIdx.x % LANES) * N, Hq = P.q.H;
  const Side sq = P.q, sk = P.k;
  auto at = [&](const Row& r, const char*& src, char*& dst, int& side) {
    side = r.h >= Hq;
    const Pick X = pick(side, sq, sk);
    const size_t t = t0 + r.tl, in = ((r.h - (side ? Hq : 0)) * D + i0) * sizeof(T);
    src = X.x + t * X.xs + in;
    dst = X.out + t * X.outs + in;
  };
  Row r{0, 0}, n;
  r.next((int)threadIdx.x / LANES, H);
  const char* src; char* dst; int side = 0;
  u32x4 lo = {0, 0, 0, 0}, hi = {0, 0, 0, 0};
  if (r.tl < nt) {
    at(r, src, dst, side);
    lo = load16<PAST>(src);
    hi = load16<PAST>(src + D / 2 * sizeof(T));
  }
  load_weights(P, S);
  load_angles(P, S, t0, nt);
  __syncthreads();
  while (r.tl < nt) {
    n = r;
    n.next(ROWS, H);
    const char* nsrc; char* ndst = nullptr; int nside = 0;
    u32x4 nlo = lo, nhi = hi;
    if (n.tl < nt) {
      at(n, nsrc, ndst, nside);
      nlo = load16<PAST>(nsrc);
      nhi = load16<PAST>(nsrc + D / 2 * sizeof(T));
    }
    float a[N], b[N], c[N], s[N];
    Vec<T>::get(lo, a);
    Vec<T>::get(hi, b);
    if (side ? sk.w != nullptr : sq.w != nullptr) {
      float sq = 0.f, wa[N], wb[N];
#pragma unroll
      for (int x = 0; x < N; ++x) sq = fmaf(a[x], a[x], fmaf(b[x], b[x], sq));
      const float rs = 1.f / __fsqrt_rn(head_sum<LANES>(sq) * (1.f / D) + P.eps);
      lds_get(&S.w[side][i0], wa);
      lds_get(&S.w[side][i0 + D / 2], wb);
#pragma unroll
      for (int x = 0; x < N; ++x) {
        a[x] = a[x] * rs * wa[x];
        b[x] = b[x] * rs * wb[x];
      }
    }
    lds_get(&S.cs[r.tl][i0], c);
    lds_get(&S.sn[r.tl][i0], s);
    float ya[N], yb[N];
#pragma unroll
    for (int x = 0; x < N; ++x) {
      ya[x] = fmaf(a[x], c[x], -(b[x] * s[x]));
      yb[x] = fmaf(b[x], c[x], a[x] * s[x]);
    }
    store16(dst, Vec<T>::put(ya));
    store16(dst + D / 2 * sizeof(T), Vec<T>::put(yb));
    r = n; lo = nlo; hi = nhi; dst = ndst; side = nside;
  }
}

template <typename T, int D, int TB, bool PAST>
__global__ void __launch_bounds__(NT) qk_norm_rope_grad_kernel(const Params P) {
  constexpr int N = Vec<T>::N, LANES = D / 2 / N, ROWS = NT / LANES;
  __shared__ Shared<D, TB> S;
  __shared__ float red[NT / 64][2][D];
  const int H = P.q.H + P.k.H, lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  const int i0 = (threadIdx.x % LANES) * N, Hq = P.q.H;
  const Side sq = P.q, sk = P.k;
  float dwa[2][N], dwb[2][N];                               // of queries and keys
#pragma unroll
  for (int x = 0; x < N; ++x) dwa[0][x] = dwa[1][x] = dwb[0][x] = dwb[1][x] = 0.f;
  load_weights(P, S);
  const int blocks = (P.T + TB - 1) / TB;
  for (int blk = blockIdx.x; blk < blocks; blk += gridDim.x) {
    const int t0 = blk * TB, nt = min(TB, P.T - t0);
    auto offset = [&](const Row& r, int side) { return (size_t)(((r.h - (side ? Hq : 0)) * D + i0) * sizeof(T)); };
    u32x4 v[4] = {};                                        // x, dy: lower and upper half
    auto fetch = [&](const Row& r, int& side) {
      side = r.h >= Hq;
      const Pick X = pick(side, sq, sk);
      const size_t t = t0 + r.tl, in = offset(r, side);
      const char* const dy = X.dy + t * X.dys + in;
      v[2] = load16<PAST>(dy);
      v[3] = load16<PAST>(dy + D / 2 * sizeof(T));
      if (X.norm) {
        const char* const x = X.x + t * X.xs + in;
        v[0] = load16<PAST>(x);
        v[1] = load16<PAST>(x + D / 2 * sizeof(T));
      }
    };
    Row r{0, 0};
    r.next((int)threadIdx.x / LANES, H);
    int side = 0;
    if (r.tl < nt) fetch(r, side);
    __syncthreads();                                        // the angles of the block before are used up
    load_angles(P, S, t0, nt);
    __syncthreads();
    while (r.tl < nt) {
      float xa[N], xb[N], ga[N], gb[N], c[N], s[N];
      Vec<T>::get(v[0], xa);
      Vec<T>::get(v[1], xb);
      Vec<T>::get(v[2], ga);
      Vec<T>::get(v[3], gb);
      const Row now = r;
      const int now_side = side;
      r.next(ROWS, H);
      if (r.tl < nt) fetch(r, side);
      lds_get(&S.cs[now.tl][i0], c);
      lds_get(&S.sn[now.tl][i0], s);
#pragma unroll
      for (int x = 0; x < N; ++x) {
        const float l = ga[x], h = gb[x];
        ga[x] = fmaf(l, c[x], h * s[x]);
        gb[x] = fmaf(h, c[x], -(l * s[x]));
      }
      const Pick X = pick(now_side, sq, sk);
      if (X.norm) {
        float sq = 0.f, dot = 0.f, wa[N], wb[N];
        lds_get(&S.w[now_side][i0], wa);
        lds_get(&S.w[now_side][i0 + D / 2], wb);
#pragma unroll
        for (int x = 0; x < N; ++x) sq = fmaf(xa[x], xa[x], fmaf(xb[x], xb[x], sq));
        const float rs = 1.f / __fsqrt_rn(head_sum<LANES>(sq) * (1.f / D) + P.eps);
        const int other = now_side;
#pragma unroll
        for (int x = 0; x < N; ++x) {
          xa[x] *= rs;
          xb[x] *= rs;
          const float da = ga[x] * xa[x], db = gb[x] * xb[x];
          if (other) { dwa[1][x] += da; dwb[1][x] += db; } else { dwa[0][x] += da; dwb[0][x] += db; }
          ga[x] *= wa[x];
          gb[x] *= wb[x];
          dot = fmaf(ga[x], xa[x], fmaf(gb[x], xb[x], dot));
        }
        const float m = head_sum<LANES>(dot) * (1.f / D);
#pragma unroll
        for (int x = 0; x < N; ++x) {
          ga[x] = rs * fmaf(-xa[x], m, ga[x]);
          gb[x] = rs * fmaf(-xb[x], m, gb[x]);
        }
      }
      char* const dst = X.out + (size_t)(t0 + now.tl) * X.outs + offset(now, now_side);
      store16(dst, Vec<T>::put(ga));
      store16(dst + D / 2 * sizeof(T), Vec<T>::put(gb));
    }
  }
  if (!P.part) return;
#pragma unroll
  for (int sd = 0; sd < 2; ++sd)
#pragma unroll
    for (int x = 0; x < N; ++x) {
#pragma unroll
      for (int o = LANES; o < 64; o <<= 1) {
        dwa[sd][x] += __shfl_xor(dwa[sd][x], o, 64);
        dwb[sd][x] += __shfl_xor(dwb[sd][x], o, 64);
      }
      if (lane < LANES) {
        red[wv][sd][i0 + x] = dwa[sd][x];
        red[wv][sd][i0 + D / 2 + x] = dwb[sd][x];
      }
    }
  __syncthreads();
  for (int x = threadIdx.x; x < 2 * D; x += NT) {
    const float* const p = &red[0][0][0] + x;
    P.part[(size_t)blockIdx.x * 2 * D + x] = p[0] + p[2 * D] + p[4 * D] + p[6 * D];
  }
}

// weight gradients: column sums of part[groups][2][D], 16 columns to a workgroup, 64 threads to four of them (in fp64, eight loads at a time:
// one after the other 1024 rows of 256 columns took 21 us)
template <int D>
__global__ void __launch_bounds__(NT) qk_norm_rope_dw_kernel(const float* part, int groups, float* dqw, float* dkw) {
  __shared__ double red[64][17];
  const int cl = (threadIdx.x & 3) * 4, rl = threadIdx.x >> 2, col = blockIdx.x * 16 + cl;
  double s[4] = {0.0, 0.0, 0.0, 0.0};
  for (int g0 = 0; g0 < groups; g0 += 512) {
    float4 v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int g = g0 + 64 * i + rl;
      v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (g < groups) v[i] = *reinterpret_cast<const float4*>(part + (size_t)g * 2 * D + col);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) { s[0] += v[i].x; s[1] += v[i].y; s[2] += v[i].z; s[3] += v[i].w; }
  }
#pragma unroll
  for (int x = 0; x < 4; ++x) red[rl][cl + x] = s[x];
  __syncthreads();
  const int c = threadIdx.x & 15, q = threadIdx.x >> 4;     // 16 threads to a column
  double t = red[4 * q][c] + red[4 * q + 1][c] + red[4 * q + 2][c] + red[4 * q + 3][c];
  __syncthreads();
  red[q][c] = t;
  __syncthreads();
  if (q == 0) {
    for (int x = 1; x < 16; ++x) t += red[x][c];
    const int column = blockIdx.x * 16 + c;
    float* const out = column < D ? dqw : dkw;
    if (out) out[column < D ? column : column - D] = (float)t;
  }
}

int check(int dtype, int64_t T, int Hq, int Hkv, int d, const int32_t* sections, float eps) {
  if (T < 0 || Hq <= 0 || Hkv <= 0 || d <= 0 || !(eps >= 0.f) || eps > 3.0e38f) return -1;
  if ((dtype != 0 && dtype != 1) || (d != 64 && d != 128) || T > 0x7FFFFFFF - 64) return -2;
  if (Hq > (1 << 20) || Hkv > (1 << 20)) return -2;
  if (sections[0] < 0 || sections[1] < 0 || sections[2] < 0 || (int64_t)sections[0] + sections[1] + sections[2] != d / 2) return -2;
  return 0;
}
// a tensor of H heads a token: stride (elements) and base on 16-byte lines
bool lies(const void* p, int64_t stride, int H, int d, int e, int64_t T) {
  if ((uintptr_t)p & 15u) return false;
  if (stride % (16 / e) != 0 || stride < 0 || stride > ((int64_t)1 << 40)) return false;
  return T <= 1 || stride >= (int64_t)H * d;
}
int groups_for(int64_t T, int TB) {
  const int64_t blocks = (T + TB - 1) / TB;
  return (int)(blocks < MAX_GROUPS ? blocks : MAX_GROUPS);
}
// Tokens a workgroup takes: with four, its 64 angles each keep all threads busy once.
int tokens_per_group(int64_t T) { return T > 1024 ? 4 : 1; }

// [fp32, bf16][64, 128 columns][form]
#define RLNR_KERNELS(kernel)                                                                                            \
  {{{kernel<float, 64, 1, false>, kernel<float, 64, 4, false>, kernel<float, 64, 4, true>},                             \
    {kernel<float, 128, 1, false>, kernel<float, 128, 4, false>, kernel<float, 128, 4, true>}},                         \
   {{kernel<__bf16, 64, 1, false>, kernel<__bf16, 64, 4, false>, kernel<__bf16, 64, 4, true>},                          \
    {kernel<__bf16, 128, 1, false>, kernel<__bf16, 128, 4, false>, kernel<__bf16, 128, 4, true>}}}
constexpr int64_t CACHED = (int64_t)192 << 20;              // bytes read; the last-level cache has 256 MB
int form(int TB, int64_t bytes) { return TB == 1 ? 0 : bytes <= CACHED ? 1 : 2; }
template <typename Desc> int64_t Hq_Hkv(const Desc* d) { return (int64_t)d->Hq + d->Hkv; }

int check_backward(const rl_qk_norm_rope_backward_desc* d) {
  if (!d) return -1;
  if (d->struct_size != sizeof(rl_qk_norm_rope_backward_desc)) return -4;
  return check(d->dtype, d->T, d->Hq, d->Hkv, d->d, d->sections, d->eps);
}
size_t bytes_for(const rl_qk_norm_rope_backward_desc* d) {
  if (!d->q_weight && !d->k_weight) return 0;
  return (size_t)groups_for(d->T, tokens_per_group(d->T)) * 2 * d->d * sizeof(float);
}

}  // namespace

extern "C" {

int rl_qk_norm_rope(const rl_qk_norm_rope_desc* d, void* hip_stream) {
  if (!d) return -1;
  if (d->struct_size != sizeof(rl_qk_norm_rope_desc)) return -4;
  const int rc = check(d->dtype, d->T, d->Hq, d->Hkv, d->d, d->sections, d->eps);
  if (rc != 0) return rc;
  if (d->T == 0) return 0;
  if (!d->q || !d->k || !d->positions || !d->inv_freq || !d->q_out || !d->k_out) return -1;
  const int e = d->dtype == 0 ? 4 : 2;
  if (!lies(d->q, d->q_stride, d->Hq, d->d, e, d->T) || !lies(d->k, d->k_stride, d->Hkv, d->d, e, d->T) ||
      !lies(d->q_out, d->q_out_stride, d->Hq, d->d, e, d->T) || !lies(d->k_out, d->k_out_stride, d->Hkv, d->d, e, d->T)) return -2;
  Params P{};
  P.q = Side{static_cast<const char*>(d->q), nullptr, static_cast<char*>(d->q_out), d->q_weight, d->Hq, d->q_stride * e, 0, d->q_out_stride * e};
  P.k = Side{static_cast<const char*>(d->k), nullptr, static_cast<char*>(d->k_out), d->k_weight, d->Hkv, d->k_stride * e, 0, d->k_out_stride * e};
  P.pos = d->positions; P.inv_freq = d->inv_freq;
  P.T = (int)d->T; P.s0 = d->sections[0]; P.s1 = d->sections[1]; P.eps = d->eps;
  typedef void (*kern_t)(const Params);
  static constexpr kern_t kerns[2][2][3] = RLNR_KERNELS(qk_norm_rope_kernel);
  const int TB = tokens_per_group(d->T);
  const int64_t blocks = (d->T + TB - 1) / TB;
  const dim3 grid((unsigned)(blocks < GRID_X ? blocks : GRID_X), (unsigned)((blocks + GRID_X - 1) / GRID_X));
  hipLaunchKernelGGL(kerns[d->dtype][d->d == 128][form(TB, Hq_Hkv(d) * d->T * d->d * e)], grid, dim3(NT), 0, static_cast<hipStream_t>(hip_stream), P);
  return hipGetLastError() == hipSuccess ? 0 : -5;
}

size_t rl_qk_norm_rope_backward_workspace_bytes(const rl_qk_norm_rope_backward_desc* d) {
  return check_backward(d) == 0 ? bytes_for(d) : 0;
}

int rl_qk_norm_rope_backward(const rl_qk_norm_rope_backward_desc* d, void* hip_stream) {
  const int rc = check_backward(d);
  if (rc != 0) return rc;
  if ((d->q_weight && !d->dq_weight) || (d->k_weight && !d->dk_weight)) return -1;
  const size_t need = bytes_for(d);
  if (d->T > 0) {
    if (!d->dq_out || !d->dk_out || !d->positions || !d->inv_freq || !d->dq || !d->dk) return -1;
    if ((d->q_weight && !d->q) || (d->k_weight && !d->k)) return -1;
    const int e = d->dtype == 0 ? 4 : 2;
    if (!lies(d->dq_out, d->dq_out_stride, d->Hq, d->d, e, d->T) || !lies(d->dk_out, d->dk_out_stride, d->Hkv, d->d, e, d->T) ||
        !lies(d->dq, d->dq_stride, d->Hq, d->d, e, d->T) || !lies(d->dk, d->dk_stride, d->Hkv, d->d, e, d->T)) return -2;
    if ((d->q_weight && !lies(d->q, d->q_stride, d->Hq, d->d, e, d->T)) || (d->k_weight && !lies(d->k, d->k_stride, d->Hkv, d->d, e, d->T))) return -2;
    if (need > 0 && (!d->workspace || d->workspace_bytes < need || ((uintptr_t)d->workspace & 255u))) return -3;
  }
  const int e = d->dtype == 0 ? 4 : 2;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  Params P{};
  P.q = Side{static_cast<const char*>(d->q), static_cast<const char*>(d->dq_out), static_cast<char*>(d->dq), d->q_weight, d->Hq,
             d->q_stride * e, d->dq_out_stride * e, d->dq_stride * e};
  P.k = Side{static_cast<const char*>(d->k), static_cast<const char*>(d->dk_out), static_cast<char*>(d->dk), d->k_weight, d->Hkv,
             d->k_stride * e, d->dk_out_stride * e, d->dk_stride * e};
  P.pos = d->positions; P.inv_freq = d->inv_freq;
  P.T = (int)d->T; P.s0 = d->sections[0]; P.s1 = d->sections[1]; P.eps = d->eps;
  P.part = need > 0 ? static_cast<float*>(d->workspace) : nullptr;
  typedef void (*kern_t)(const Params);
  static constexpr kern_t kerns[2][2][3] = RLNR_KERNELS(qk_norm_rope_grad_kernel);
  const int TB = tokens_per_group(d->T), groups = groups_for(d->T, TB);
  if (groups > 0) hipLaunchKernelGGL(kerns[d->dtype][d->d == 128][form(TB, 2 * Hq_Hkv(d) * d->T * d->d * e)], dim3(groups), dim3(NT), 0, st, P);
  if (d->q_weight || d->k_weight) {
    float* const dqw = d->q_weight ? d->dq_weight : nullptr;
    float* const dkw = d->k_weight ? d->dk_weight : nullptr;
    if (d->d == 128) hipLaunchKernelGGL((qk_norm_rope_dw_kernel<128>), dim3(16), dim3(NT), 0, st, P.part, groups, dqw, dkw);
    else             hipLaunchKernelGGL((qk_norm_rope_dw_kernel<64>), dim3(8), dim3(NT), 0, st, P.part, groups, dqw, dkw);
  }
  return hipGetLastError() == hipSuccess ? 0 : -5;
}

}  // extern "C"
