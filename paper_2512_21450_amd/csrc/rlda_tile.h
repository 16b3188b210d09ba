// A tile of a bf16 matrix product on the matrix cores, C[m, n] = sum_k A(m, k) B(n, k), fp32 sums in registers.
//
// An operand is a matrix of rows and columns in memory whose contraction index k runs along its columns (K_COLS: the rows are
// m or n) or along its rows (K_ROWS: the columns are m or n).  Tiles of BK k move from memory straight into LDS (16 bytes a
// lane, a wavefront's 1 KB lands contiguously) into a ring of STAGES buffers, all but one ahead of the products.  Tiles of 256 take two of 64 k:
// four of 32 k, lines of 64 bytes, made 4096 x 151936 x 3584 5 % slower (4.07 -> 4.30 ms); fragments asked for a step ahead (4.07) and
// wavefronts of a SIMD that fetch and multiply in turns between barriers (4.05 to 4.2) gained nothing, one wavefront a SIMD with 128 x 128 lost (4.6);
// the forward call's product takes 3.8 ms now, and the card holds 1.65 GHz at 59 % of the matrix unit's cycles under this load.  Tiles of few rows, whose loads are all there is to do,
// take four buffers (16 x 151936 x 2048: 137 us with two, 118 with four, 130 with eight).  The
// layout's xor pattern, under which fragment reads meet no bank conflict, is applied to the lane's address in memory: K_COLS fragments are read with
// 16-byte reads (16 rows at one column must differ), K_ROWS fragments with the transposing 8-byte reads (4 rows of 64 bytes each).
// Products are 32x32x16: lane l holds column n = l % 32 of C, and rows m = 8 (x / 4) + 4 (l / 32) + x % 4 in its 16 registers.
//
// The loads into LDS are asm: the compiler, which cannot tell what bytes they write, would otherwise let every LDS read wait for
// all of them.  What orders them is written out: a wavefront waits for its own, then all meet at a barrier.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace rlda {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

#define RLDA_AS3(T, addr) ((__attribute__((address_space(3))) T*)(uintptr_t)(addr))

// M0 is the compiler's to set before each instruction of its own that reads it; it keeps nothing there in between.
// 64 lanes x 16 bytes from base + offset (unsigned, per lane) to LDS at `lds` (uniform) + 16 * lane
__device__ __forceinline__ void load_to_lds(const char* base, uint32_t offset, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(offset), "s"(base));
}
// all but the last PENDING of this wavefront's loads have landed and its LDS reads are done; then everybody's
template <int PENDING = 0>
__device__ __forceinline__ void landed_barrier() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(PENDING) : "memory");
}

// LDS writes of all wavefronts are there
__device__ __forceinline__ void written_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

enum Layout { K_COLS, K_ROWS };

// one operand's tile of R (m or n) by BK; `ld2`: bytes between rows in memory
template <Layout L, int R, int WAVES, int BK>
struct Operand {
  static constexpr int BYTES = R * BK * 2, LOADS = BYTES / 1024 / WAVES;
  static constexpr int ROWB = L == K_COLS ? BK * 2 : R * 2, CHUNKS = ROWB / 16, ROWS_PER_LOAD = 64 / CHUNKS;
  static_assert(BYTES % (1024 * WAVES) == 0, "whole loads per wavefront");
  __device__ static __forceinline__ int pattern(int row) { return L == K_ROWS ? (row & 3) << 2 : BK == 64 ? (row >> 1) & 7 : (row >> 2) & 3; }

  const char* base;                                         // of the tile's first row or column, at k = 0
  uint32_t offset[LOADS];                                   // per lane
  int64_t step;                                             // bytes per BK
  uint32_t ld2;

  // rows (K_COLS) from `at` on, of which `live` exist, or columns (K_ROWS): what lies past them reads the last one again
  __device__ __forceinline__ void init(const void* p, int64_t ld, int64_t at, int64_t live, int wv, int lane) {
    ld2 = (uint32_t)(ld * 2);
    base = static_cast<const char*>(p) + (L == K_COLS ? at * ld * 2 : at * 2);
    step = L == K_COLS ? BK * 2 : (int64_t)BK * ld * 2;
    const int last = (int)((live - at < R ? live - at : R) - 1);
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int row = (wv * LOADS + i) * ROWS_PER_LOAD + lane / CHUNKS, chunk = (lane % CHUNKS) ^ pattern(row);
      offset[i] = L == K_COLS ? (uint32_t)min(row, last) * ld2 + chunk * 16 : (uint32_t)row * ld2 + min(chunk, last / 8) * 16;
    }
  }
  // the loads of k-step kt; only the first `exist` 16-byte chunks of a row's BK (K_COLS) or `exist` rows (K_ROWS) exist: the others
  // read the last one, and clear() puts zeros over it once it has landed (zeros of the other operand would not do: 0 * infinity is not 0)
  template <bool FULL>
  __device__ __forceinline__ void issue(int kt, uint32_t lds, int wv, int lane, int exist) const {
    const char* const from = base + kt * step;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      uint32_t o = offset[i];
      if constexpr (!FULL) {
        const int row = (wv * LOADS + i) * ROWS_PER_LOAD + lane / CHUNKS;
        if constexpr (L == K_COLS) {
          const int chunk = (lane % CHUNKS) ^ pattern(row);
          o -= (uint32_t)(chunk - min(chunk, exist - 1)) * 16;
        } else {
          o -= (uint32_t)(row - min(row, exist - 1)) * ld2;
        }
      }
      load_to_lds(from, o, lds + (wv * LOADS + i) * 1024);
    }
  }
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  __device__ __forceinline__ void clear(uint32_t lds, int wv, int lane, int exist) const {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int row = (wv * LOADS + i) * ROWS_PER_LOAD + lane / CHUNKS;
      if ((L == K_COLS ? (lane % CHUNKS) ^ pattern(row) : row) >= exist) *RLDA_AS3(u32x4, lds + (wv * LOADS + i) * 1024 + lane * 16) = u32x4{0, 0, 0, 0};
    }
  }
  // zeros in place of infinities and NaN
  __device__ __forceinline__ void tidy(uint32_t lds, int wv, int lane) const {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      u32x4 v = *RLDA_AS3(const u32x4, lds + (wv * LOADS + i) * 1024 + lane * 16);
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const uint32_t lo = (v[x] & 0x7F80u) == 0x7F80u ? 0u : 0xFFFFu, hi = (v[x] & 0x7F800000u) == 0x7F800000u ? 0u : 0xFFFF0000u;
        v[x] &= lo | hi;
      }
      *RLDA_AS3(u32x4, lds + (wv * LOADS + i) * 1024 + lane * 16) = v;
    }
  }
};

// fragments of TILES blocks of 32 (m or n) from row / column `first` of the tile on
template <typename O, Layout L, int TILES, int BK>
struct Fragments {
  static constexpr int ROWB = O::ROWB;
  uint32_t at[L == K_COLS ? BK / 16 : TILES];
  __device__ __forceinline__ void init(int first, int lane) {
    if constexpr (L == K_COLS) {
      const int row = first + (lane & 31);
#pragma unroll
      for (int ks = 0; ks < BK / 16; ++ks) at[ks] = row * ROWB + (((2 * ks + (lane >> 5)) ^ O::pattern(row)) << 4);
    } else {
      const int m16 = lane & 15, row = 8 * (lane >> 5) + (m16 >> 2);
#pragma unroll
      for (int t = 0; t < TILES; ++t) {
        const int chunk = first / 8 + 4 * t + 2 * ((lane >> 4) & 1) + ((m16 & 3) >> 1);
        at[t] = row * ROWB + ((chunk ^ O::pattern(row)) << 4) + ((m16 & 1) << 3);
      }
    }
  }
  __device__ __forceinline__ bf16x8 get(uint32_t lds, int ks, int t) const {
    if constexpr (L == K_COLS) {
      return *RLDA_AS3(const bf16x8, lds + at[ks] + t * 32 * ROWB);
    } else {
      union { s16x4 h[2]; bf16x8 v; } f;
      f.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(RLDA_AS3(s16x4, lds + at[t] + ks * 16 * ROWB));
      f.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(RLDA_AS3(s16x4, lds + at[t] + (ks * 16 + 4) * ROWB));
      return f.v;
    }
  }
};

// WM x WN wavefronts, each MT x NT blocks of 32 x 32
template <int WM_, int WN_, int MT_, int NT_, int BK_, int STAGES_, Layout LA, Layout LB>
struct Tile {
  static constexpr int WM = WM_, WN = WN_, MT = MT_, NT = NT_, BK = BK_, STAGES = STAGES_, WAVES = WM * WN, THREADS = 64 * WAVES;
  static constexpr int BM = WM * MT * 32, BN = WN * NT * 32;
  static_assert((STAGES & (STAGES - 1)) == 0, "a power of two");
  typedef Operand<LA, BM, WAVES, BK> OA;
  typedef Operand<LB, BN, WAVES, BK> OB;
  static constexpr int STAGE = OA::BYTES + OB::BYTES, LDS = STAGES * STAGE;

  // k-steps [k0, k1); `tail`: 16-byte chunks (K_COLS) or rows (K_ROWS) that A has in step tail_step.  MAY_TIDY and `tidy`: A's infinities and NaN
  // count as zeros.
  template <bool MAY_TIDY = false>
  __device__ static __forceinline__ void run(const OA& a, const OB& b, int k0, int k1, int tail_step, int tail, uint32_t lds,
                                             f32x16 (&acc)[MT][NT], bool tidy = false) {
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wv % WM, wn = wv / WM;
    Fragments<OA, LA, MT, BK> fa;
    Fragments<OB, LB, NT, BK> fb;
    fa.init(wm * MT * 32, lane);
    fb.init(wn * NT * 32, lane);
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int x = 0; x < 16; ++x) acc[i][j][x] = 0.f;
    auto issue = [&](int kt) {
      const uint32_t to = lds + ((kt - k0) & (STAGES - 1)) * STAGE;
      if (kt == tail_step) a.template issue<false>(kt, to, wv, lane, tail);
      else                 a.template issue<true>(kt, to, wv, lane, 0);
      b.template issue<true>(kt, to + OA::BYTES, wv, lane, 0);
    };
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i)
      if (k0 + i < k1) issue(k0 + i);
    for (int kt = k0; kt < k1; ++kt) {
      // step kt is there, and nobody reads the buffer of the one before any more
      if (kt + STAGES - 2 < k1) landed_barrier<(STAGES - 2) * (OA::LOADS + OB::LOADS)>();
      else                      landed_barrier();
      if (kt + STAGES - 1 < k1) issue(kt + STAGES - 1);
      const uint32_t cur = lds + ((kt - k0) & (STAGES - 1)) * STAGE;
      if (kt == tail_step) {
        a.clear(cur, wv, lane, tail);
        written_barrier();
      }
      if constexpr (MAY_TIDY) {
        if (tidy) {
          a.tidy(cur, wv, lane);
          written_barrier();
        }
      }
#pragma unroll
      for (int ks = 0; ks < BK / 16; ++ks) {
        bf16x8 af[MT], bf[NT];
#pragma unroll
        for (int i = 0; i < MT; ++i) af[i] = fa.get(cur, ks, i);
#pragma unroll
        for (int j = 0; j < NT; ++j) bf[j] = fb.get(cur + OA::BYTES, ks, j);
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int i = 0; i < MT; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(af[i], bf[j], acc[i][j], 0, 0, 0);
      }
    }
    landed_barrier();                                       // the buffers are free
  }
};

}  // namespace
}  // namespace rlda
