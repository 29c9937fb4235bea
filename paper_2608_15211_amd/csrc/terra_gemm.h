// terra_gemm.h - what the matrix-core products of the Swin block (block.hip)
// and of the linear layer (linear.hip) share: XOR-swizzled LDS tiles, their
// direct-to-LDS staging, the operand reads, and GELU.
//
// Operands are row-major matrices of 16-bit elements in HBM.  A matrix of
// 8-bit elements whose contraction index runs along memory rows is staged as
// one of half as many 16-bit elements: the tiles hold the same bytes.
#pragma once

#include "terra_common.h"

namespace terra {

typedef __bf16 bf16;
typedef short v4s __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4s lds_v4s;

constexpr int kBM = 256;          // rows and columns of a workgroup tile, eight-wave form
constexpr int kBS = 128;          // four-wave form
constexpr int kBK = 64;           // contraction depth per stage
constexpr int kEpiS = 68;         // row stride (floats) of a wave's epilogue staging tile

// A 16-bit operand in memory: row-major, `ld` elements a row, `rows` valid rows.
struct Mat {
  const bf16* p;
  int ld;
  int rows;
  // Three-part operand (read only by SEG kernels): three [rows][segw]
  // matrices side by side, part i at element offset i * segstride from p.
  int segw;
  int64_t segstride;
  __device__ const bf16* at(int r, int c) const { return p + (int64_t)r * ld + c; }
};

// Phi(x), the standard normal distribution function: with a = |x|,
// Phi(-a) = 2^P(a), P a degree-8 polynomial fitted to log2 Phi(-a) on
// [0, 5.6] (weighted minimax; P falls without bound beyond, where Phi(-a) <
// 1.1e-8).  Largest error as the hardware computes it, over 5e6 points from
// -40 to 40: Phi 5.7e-8 below zero and 8.2e-8 above (one minus it), GELU
// 4.0e-7, its derivative 1.3e-7.  One exponential and no division: the MLP
// epilogues are bound by vector instructions.  Against Abramowitz and
// Stegun's 7.1.26 (a reciprocal and an exponential: 2.9e-7, 4.7e-7 and 3.2e-7
// on the same points, and no interval where it is closer) the fc1 epilogue
// goes from 21.6 to 17.6 instructions an element and the 128 x 1080 fc1
// product from 1026 to 959 us, dh from 890 to 851.
__device__ inline float phi_f(float x) {
  const float a = fabsf(x);
  float p = -2.772049e-06f;
  p = fmaf(p, a, 3.8620746e-05f);
  p = fmaf(p, a, -1.8254759e-04f);
  p = fmaf(p, a, -1.4587014e-04f);
  p = fmaf(p, a, 7.0754718e-03f);
  p = fmaf(p, a, -5.2505028e-02f);
  p = fmaf(p, a, -0.45920491f);
  p = fmaf(p, a, -1.1511058f);
  p = fmaf(p, a, -1.0f);
  const float w = __builtin_amdgcn_exp2f(p);
  return x > 0.0f ? 1.0f - w : w;
}
__device__ inline float gelu_f(float x) { return x * phi_f(x); }
// Phi(x) + x phi(x), phi(x) = 2^(-x^2 log2(e) / 2 - log2(sqrt(2 pi)))
__device__ inline float gelu_grad_f(float x) {
  return fmaf(x, __builtin_amdgcn_exp2f(fmaf(x * x, -0.72134752f, -1.3257481f)), phi_f(x));
}

// ---------------------------------------------------------------------------
// LDS tiles.  A stage holds the A tile (kBM output rows x kBK) and the B tile
// (kBN x kBK), each in its memory layout, unpadded, with the 16-byte chunks
// of each row permuted by an XOR of the row index so that the matrix-core
// operand reads hit distinct banks:
// * KROW tile (memory [R][BK], BK / 8 chunks a row): chunk c of row r sits at
//   chunk c ^ ((r >> 1) & 7) - 16 consecutive rows read at one logical chunk
//   cover all 64 banks;
// * COLK tile (memory [BK][R], R / 8 chunks a row): chunk c of row k sits
//   at chunk c ^ (4 (k & 3)) - each half-wave of a transpose read takes 64
//   bytes from each of four rows, and these land on four different 64-byte
//   spans of the 256 bytes the LDS banks cover (measured: no bank conflicts;
//   with c ^ (2 (k & 3)) 0.8-2 conflict cycles per LDS instruction, though
//   no slower).
// ---------------------------------------------------------------------------
template <int R, bool KROW, int BK, int NT = 512>
struct Tile {
  static constexpr int kChunks = R * BK / 8;    // 16-byte chunks
  static constexpr int kPer = kChunks / NT;     // per thread (NT threads)
  static constexpr int kElems = R * BK;
  static constexpr int kCpr = BK / 8;           // chunks a row (KROW)
  __device__ static int swz(int row) { return (row >> 1) & 7; }
  // element offset of (row, logical chunk) of the memory layout
  __device__ static int off(int row, int c) {
    if (KROW) return row * BK + 8 * (c ^ swz(row));
    return row * R + 8 * (c ^ (4 * (row & 3)));
  }
  // memory (row, column) of the chunk stored in slot q (slot = chunk position in LDS order)
  __device__ static void slot_src(int q, int r0, int k0, int& mrow, int& mcol) {
    if (KROW) {
      const int row = q / kCpr, p = q % kCpr;
      mrow = r0 + row;
      mcol = k0 + 8 * (p ^ swz(row));
    } else {
      const int row = q / (R / 8), p = q - row * (R / 8);
      mrow = k0 + row;
      mcol = r0 + 8 * (p ^ (4 * (row & 3)));
    }
  }
};

// Straight operand (KROW tile): lane l receives T[m0 + l % 32][k0 + 8h + x],
// x = 0..7, h = l / 32, as one 16-byte read.
template <int R, int BK>
__device__ inline bf16x8 row_operand(const bf16* T, int k0, int m0, int lane) {
  const int row = m0 + (lane & 31);
  return *reinterpret_cast<const bf16x8*>(T + Tile<R, true, BK>::off(row, (k0 >> 3) + (lane >> 5)));
}

// Natural-order transposed operand (COLK tile): lane l receives
// T[k0 + 8h + x][m0 + l % 32], x = 0..7.  In each 16-lane group G of the
// transpose read, lane i gets element i % 4 of the 8 bytes that lane
// 16G + 4x + i/4 addresses, so lane L addresses row k0 + 8h + (L % 16) / 4
// (4 rows further for the second read), columns m0 + 16 (G % 2) + 4 (L % 4).
template <int R, int BK>
__device__ inline bf16x8 tr_operand(const bf16* T, int k0, int m0, int lane) {
  const int G = lane >> 4;
  const int row = k0 + 8 * (G >> 1) + ((lane & 15) >> 2);
  const int m = m0 + 16 * (G & 1) + 4 * (lane & 3);
  const int c = m >> 3, e = m & 7;
  const bf16* p0 = T + Tile<R, false, BK>::off(row, c) + e;
  const bf16* p1 = T + Tile<R, false, BK>::off(row + 4, c) + e;
  const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)p0);
  const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)p1);
  typedef short v8s __attribute__((ext_vector_type(8)));
  const v8s o = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
  return __builtin_bit_cast(bf16x8, o);
}

// Direct-to-LDS staging of one operand tile: each thread moves kPer 16-byte
// chunks with buffer loads that write LDS themselves (slot q of the tile is
// written by thread q % NT, load q / NT); chunks outside the operand or the
// contraction slice read zeros.  The per-thread part of each chunk's address
// does not change along the contraction, so it is worked out once (init) and
// a stage costs one add and one bounds select a load.  KROW: the contraction
// index runs along memory rows.
template <int R, bool KROW, int BK, int NT>
struct Stager {
  typedef Tile<R, KROW, BK, NT> T;
  int voff[T::kPer];   // byte offset at contraction index 0 (2^31: outside the operand)
  int kpos[T::kPer];   // the chunk's contraction index inside a stage
  __device__ void init(const Mat& X, int r0, int nouter, int64_t base) {
#pragma unroll
    for (int u = 0; u < T::kPer; ++u) {
      int mr, mc;
      T::slot_src(u * NT + threadIdx.x, r0, 0, mr, mc);
      kpos[u] = KROW ? mc : mr;
      const bool ok = (KROW ? mr : mc) < nouter;
      voff[u] = ok ? (int)((base + (int64_t)mr * X.ld + mc) * 2) : (int)0x80000000;
    }
  }
  // koff: byte offset of the stage's first contraction index; krem:
  // contraction indices left from there
  __device__ void load(const i32x4& rs, bf16* tile, int koff, int krem) const {
    static_assert(T::kPer == 4, "one group of four loads");
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);   // uniform: the LDS base goes to M0
    int v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) v[u] = kpos[u] < krem ? voff[u] + koff : (int)0x80000000;
    buffer_load_lds16x4<16 * NT>(rs, tile + 8 * wave * 64, v);   // wave-uniform bases of 64 slots
  }
};

}  // namespace terra
