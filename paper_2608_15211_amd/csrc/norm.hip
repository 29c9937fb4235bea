// norm.hip - root-mean-square norm with the residual's addition, forward (in
// the element type or in e4m3 with one scale a row) and backward.
//
//   z = x + res,  rstd = 1 / sqrt(mean(z^2) + eps),  y = gain z rstd
//   q = e4m3(y / s),  s = max(max |y| / 448, 2^-126)
// z, its squares and y stay in float32; every output is rounded once, z too:
// the norm is that of the sum before z is rounded.  Backward, with
// zh = z rstd and g = dy gain, the stored z and dz the gradient that reaches z
// by the residual stream:
//   dx = rstd (g - zh mean(g zh)) + dz,   dgain = sum over rows of dy zh
// dx is the gradient of x and of res alike.
//
// What bounds it: HBM, a row is read once and stays in registers.  A row is
// held by TPR threads (one wave, 256, 512 or, forward, 1024 threads), thread t with the
// 8-element chunks t, t + TPR, ... (NCH of them); longer rows are read again.
#include <algorithm>

#include "terra_vec.h"
#include "terra_ops.h"

namespace terra {

namespace {

// Sum and maximum over a wave, in every lane.
__device__ inline float lanes_sum(float x) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) x += __shfl_xor(x, o, 64);
  return x;
}
__device__ inline uint32_t lanes_max(uint32_t x) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) x = max(x, (uint32_t)__shfl_xor((int)x, o, 64));
  return x;
}

// The same over the threads that hold one row.  `red` has a slot for each
// wave; the waves' values are added in order.
template <int TPR>
__device__ inline float row_sum(float x, float* red) {
  x = lanes_sum(x);
  if (TPR == 64) return x;
  __syncthreads();                       // the last use of red is over
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
  __syncthreads();
  float s = 0.0f;
#pragma unroll
  for (int w = 0; w < TPR / 64; ++w) s += red[w];
  return s;
}
// Magnitudes as their bits: their order is that of the numbers, infinity above
// them and NaN above infinity, so that a NaN is not lost.
template <int TPR>
__device__ inline uint32_t row_max(uint32_t x, float* red) {
  x = lanes_max(x);
  if (TPR == 64) return x;
  uint32_t* r = reinterpret_cast<uint32_t*>(red);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) r[threadIdx.x >> 6] = x;
  __syncthreads();
  uint32_t s = 0;
#pragma unroll
  for (int w = 0; w < TPR / 64; ++w) s = max(s, r[w]);
  return s;
}
__device__ inline uint32_t mag(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// Scale of a row in e4m3 from the bits of its largest magnitude (a NaN stays
// one: the maximum would drop it).
__device__ inline float e4m3_scale(uint32_t amax) {
  const float s = __uint_as_float(amax) / kE4m3Max;
  return s < 1.17549435e-38f ? 1.17549435e-38f : s;
}

// The y of a row divided by its scale, |y / s| <= 448 but for rounding: the
// float32 quotient, correctly rounded (a zero's sign aside), by its residuals.  With i = 1 / s
// correctly rounded, q = y i is within 1.5 steps of it, q + (y - q s) i is one of
// its two neighbours, and the same once more has an exact residual and rounds
// correctly.  A power of two keeps the residuals of extreme scales normal (where they are not,
// q is far below e4m3's smallest).  An infinite scale leaves 0 of finite y.  15301
// x 1001 in bf16: 27.5 us; y i alone, a step of e4m3 off next to a tie, 26.6; the
// division operator 29.6.
struct E4m3Quotient {
  float k, s, inv;
  __device__ explicit E4m3Quotient(float scale) {
    k = scale > 0x1p60f ? 0x1p-70f : scale < 0x1p-60f ? 0x1p70f : 1.0f;
    s = scale * k;
    inv = 1.0f / s;
    if (inv == 0.0f) s = 0.0f;
  }
  __device__ void divide(float (&y)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float v = y[i] * k;
      float q = v * inv;
      q = fmaf(fmaf(-q, s, v), inv, q);
      y[i] = fmaf(fmaf(-q, s, v), inv, q);
    }
  }
};

template <int TPR>
struct Rows {
  static constexpr int kThreads = TPR == 64 ? 256 : TPR;
  static constexpr int kPer = kThreads / TPR;     // rows of a workgroup at a time
};

template <typename T, int TPR, int NCH, bool RAG>
__global__ __launch_bounds__(Rows<TPR>::kThreads) void rms_fwd_kernel(RmsFwd a) {
  __shared__ float red[16];
  const T* X = (const T*)a.x;
  const T* R = (const T*)a.res;
  T* Z = (T*)a.z;
  T* Y = (T*)a.y;
  const int t = threadIdx.x % TPR;
  const int64_t step = (int64_t)gridDim.x * Rows<TPR>::kPer;
  float g[NCH][8];
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
    const int col = 8 * (t + TPR * c);
    if (a.gain != nullptr) load8(a.gain + col, a.cols - col, g[c]);
    else
#pragma unroll
      for (int i = 0; i < 8; ++i) g[c][i] = 1.0f;
  }
  // a row's loads go out before the last one is worked on
  Chunk<T> x[NCH], r[NCH];
  auto fetch = [&](int64_t row) {
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      const int col = 8 * (t + TPR * c);
      x[c] = fetch8<RAG>(X + row * a.x_ld + col, a.cols - col);
    }
    if (R != nullptr) {
#pragma unroll
      for (int c = 0; c < NCH; ++c) {
        const int col = 8 * (t + TPR * c);
        r[c] = fetch8<RAG>(R + row * a.res_ld + col, a.cols - col);
      }
    }
  };
  int64_t row = (int64_t)blockIdx.x * Rows<TPR>::kPer + threadIdx.x / TPR;
  if (row < a.rows) fetch(row);
  for (; row < a.rows; row += step) {
    float z[NCH][8];
#pragma unroll
    for (int c = 0; c < NCH; ++c) widen8(x[c], z[c]);
    if (R != nullptr) {
#pragma unroll
      for (int c = 0; c < NCH; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) z[c][i] += to_float<T>(r[c].v[i]);
    }
    if (row + step < a.rows) fetch(row + step);
    float ss = 0.0f;
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i) ss = fmaf(z[c][i], z[c][i], ss);
    if (Z != nullptr) {
#pragma unroll
      for (int c = 0; c < NCH; ++c) {
        const int col = 8 * (t + TPR * c);
        put8<RAG>(Z + row * a.z_ld + col, a.cols - col, z[c]);
      }
    }
    const float rstd = 1.0f / sqrtf(row_sum<TPR>(ss, red) / (float)a.cols + a.eps);
    if (a.rstd != nullptr && t == 0) a.rstd[row] = rstd;
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i) z[c][i] = z[c][i] * rstd * g[c][i];
    if (Y != nullptr) {
#pragma unroll
      for (int c = 0; c < NCH; ++c) {
        const int col = 8 * (t + TPR * c);
        put8<RAG>(Y + row * a.y_ld + col, a.cols - col, z[c]);
      }
    }
    if (a.q != nullptr) {
      uint32_t amax = 0;
#pragma unroll
      for (int c = 0; c < NCH; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) amax = max(amax, mag(z[c][i]));
      const float s = e4m3_scale(row_max<TPR>(amax, red));
      if (t == 0) a.q_scale[row] = s;
      const E4m3Quotient by(s);
#pragma unroll
      for (int c = 0; c < NCH; ++c) {
        const int col = 8 * (t + TPR * c);
        by.divide(z[c]);
        store8_e4m3(a.q + row * a.q_ld + col, a.cols - col, z[c]);
      }
    }
  }
}

// Rows longer than the registers of a workgroup: read for the sum, once more for
// the scale of an 8-bit output and for the outputs, after the first time from the
// L2.  The scale is that of y itself: max |z gain| rstd, which the first pass could
// find, overflows where y does not (1100 x 40000 in bf16: 198 us, with that 151).
// Only the last pass writes, so that outputs in place of an input are not read again.
template <typename T>
__global__ __launch_bounds__(1024) void rms_fwd_long_kernel(RmsFwd a) {
  __shared__ float red[16];
  const T* X = (const T*)a.x;
  const T* R = (const T*)a.res;
  T* Z = (T*)a.z;
  T* Y = (T*)a.y;
  auto load_z = [&](int64_t row, int col, float (&z)[8]) {
    load8(X + row * a.x_ld + col, a.cols - col, z);
    if (R != nullptr) {
      float r[8];
      load8(R + row * a.res_ld + col, a.cols - col, r);
#pragma unroll
      for (int i = 0; i < 8; ++i) z[i] += r[i];
    }
  };
  auto times_gain = [&](int col, float rstd, float (&z)[8]) {
    float g[8] = {1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f};
    if (a.gain != nullptr) load8(a.gain + col, a.cols - col, g);
#pragma unroll
    for (int i = 0; i < 8; ++i) z[i] = z[i] * rstd * g[i];
  };
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    float ss = 0.0f;
    for (int col = 8 * threadIdx.x; col < a.cols; col += 8192) {
      float z[8];
      load_z(row, col, z);
#pragma unroll
      for (int i = 0; i < 8; ++i) ss = fmaf(z[i], z[i], ss);
    }
    const float rstd = 1.0f / sqrtf(row_sum<1024>(ss, red) / (float)a.cols + a.eps);
    float s = 1.0f;
    if (a.q != nullptr) {
      uint32_t amax = 0;
      for (int col = 8 * threadIdx.x; col < a.cols; col += 8192) {
        float y[8];
        load_z(row, col, y);
        times_gain(col, rstd, y);
#pragma unroll
        for (int i = 0; i < 8; ++i) amax = max(amax, mag(y[i]));
      }
      s = e4m3_scale(row_max<1024>(amax, red));
      if (threadIdx.x == 0) a.q_scale[row] = s;
    }
    if (a.rstd != nullptr && threadIdx.x == 0) a.rstd[row] = rstd;
    const E4m3Quotient by(s);
    for (int col = 8 * threadIdx.x; col < a.cols; col += 8192) {
      float z[8];
      load_z(row, col, z);
      if (Z != nullptr) store8(Z + row * a.z_ld + col, a.cols - col, z);
      times_gain(col, rstd, z);
      if (Y != nullptr) store8(Y + row * a.y_ld + col, a.cols - col, z);
      if (a.q != nullptr) {
        by.divide(z);
        store8_e4m3(a.q + row * a.q_ld + col, a.cols - col, z);
      }
    }
  }
}

// Backward.  Each wave (or workgroup) walks the rows one grid apart and keeps
// its share of dgain in registers; the waves of a workgroup add theirs in
// order through LDS, and the workgroup leaves one row of `part`.
template <typename T, int TPR, int NCH, bool RAG>
__global__ __launch_bounds__(Rows<TPR>::kThreads) void rms_bwd_kernel(RmsBwd a) {
  constexpr int kPer = Rows<TPR>::kPer;
  __shared__ float red[16];
  __shared__ float joint[TPR == 64 ? 8 * TPR * NCH : 1];
  const T* DY = (const T*)a.dy;
  const T* Z = (const T*)a.z;
  const T* DZ = (const T*)a.dz;
  T* DX = (T*)a.dx;
  const int t = threadIdx.x % TPR;
  const int64_t step = (int64_t)gridDim.x * kPer;
  float g[NCH][8], dg[NCH][8];
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
    const int col = 8 * (t + TPR * c);
#pragma unroll
    for (int i = 0; i < 8; ++i) { g[c][i] = 1.0f; dg[c][i] = 0.0f; }
    if (a.gain != nullptr) load8(a.gain + col, a.cols - col, g[c]);
  }
  const float inv = 1.0f / (float)a.cols;
  // a row's loads go out before the last one is worked on
  Chunk<T> dy[NCH], zz[NCH], dz[NCH];
  float rstd_next = 0.0f;
  auto fetch = [&](int64_t row) {
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      const int col = 8 * (t + TPR * c);
      dy[c] = fetch8<RAG>(DY + row * a.dy_ld + col, a.cols - col);
      zz[c] = fetch8<RAG>(Z + row * a.z_ld + col, a.cols - col);
    }
    rstd_next = a.rstd[row];
    if (DZ != nullptr && DX != nullptr) {
#pragma unroll
      for (int c = 0; c < NCH; ++c) {
        const int col = 8 * (t + TPR * c);
        dz[c] = fetch8<RAG>(DZ + row * a.dz_ld + col, a.cols - col);
      }
    }
  };
  int64_t row = (int64_t)blockIdx.x * kPer + threadIdx.x / TPR;
  if (row < a.rows) fetch(row);
  for (; row < a.rows; row += step) {
    float d[NCH][8], zh[NCH][8];
    Chunk<T> r[NCH];
    const float rstd = rstd_next;
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      widen8(dy[c], d[c]);
      widen8(zz[c], zh[c]);
      r[c] = dz[c];
    }
    if (row + step < a.rows) fetch(row + step);
    float s = 0.0f;
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        zh[c][i] *= rstd;
        dg[c][i] = fmaf(d[c][i], zh[c][i], dg[c][i]);
        d[c][i] *= g[c][i];
        s = fmaf(d[c][i], zh[c][i], s);
      }
    if (DX == nullptr) continue;
    const float m = row_sum<TPR>(s, red) * inv;
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      const int col = 8 * (t + TPR * c);
      float o[8] = {};
      if (DZ != nullptr) widen8(r[c], o);
#pragma unroll
      for (int i = 0; i < 8; ++i) o[i] = fmaf(rstd, fmaf(-zh[c][i], m, d[c][i]), o[i]);
      put8<RAG>(DX + row * a.dx_ld + col, a.cols - col, o);
    }
  }
  if (a.part == nullptr) return;
  if constexpr (kPer > 1) {
#pragma unroll 1
    for (int w = kPer - 1; w >= 0; --w) {       // the last wave first, wave 0 keeps the sum
      if ((int)(threadIdx.x / TPR) == w) {
#pragma unroll
        for (int c = 0; c < NCH; ++c)
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            float& slot = joint[(c * 8 + i) * TPR + t];
            if (w < kPer - 1) dg[c][i] += slot;
            slot = dg[c][i];
          }
      }
      __syncthreads();
    }
    if (threadIdx.x >= TPR) return;
  }
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
    const int col = 8 * (t + TPR * c);
    store8(a.part + (int64_t)blockIdx.x * a.cols + col, a.cols - col, dg[c]);
  }
}

// Rows longer than a workgroup's registers: two passes over the row, the share
// of dgain in the workgroup's own row of `part`.
template <typename T>
__global__ __launch_bounds__(1024) void rms_bwd_long_kernel(RmsBwd a) {
  __shared__ float red[16];
  const T* DY = (const T*)a.dy;
  const T* Z = (const T*)a.z;
  const T* DZ = (const T*)a.dz;
  T* DX = (T*)a.dx;
  float* part = a.part == nullptr ? nullptr : a.part + (int64_t)blockIdx.x * a.cols;
  bool first = true;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const float rstd = a.rstd[row];
    float s = 0.0f;
    for (int col = 8 * threadIdx.x; col < a.cols; col += 8192) {
      float d[8], z[8], w[8] = {};
      load8(DY + row * a.dy_ld + col, a.cols - col, d);
      load8(Z + row * a.z_ld + col, a.cols - col, z);
      if (part != nullptr) {
        if (!first) load8(part + col, a.cols - col, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = fmaf(d[i], z[i] * rstd, w[i]);
        store8(part + col, a.cols - col, w);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = 1.0f;
      if (a.gain != nullptr) load8(a.gain + col, a.cols - col, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) s = fmaf(d[i] * w[i], z[i] * rstd, s);
    }
    first = false;
    if (DX == nullptr) continue;
    const float m = row_sum<1024>(s, red) / (float)a.cols;
    for (int col = 8 * threadIdx.x; col < a.cols; col += 8192) {
      float d[8], z[8], w[8], r[8] = {};
      load8(DY + row * a.dy_ld + col, a.cols - col, d);
      load8(Z + row * a.z_ld + col, a.cols - col, z);
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = 1.0f;
      if (a.gain != nullptr) load8(a.gain + col, a.cols - col, w);
      if (DZ != nullptr) load8(DZ + row * a.dz_ld + col, a.cols - col, r);
#pragma unroll
      for (int i = 0; i < 8; ++i) r[i] = fmaf(rstd, fmaf(-(z[i] * rstd), m, d[i] * w[i]), r[i]);
      store8(DX + row * a.dx_ld + col, a.cols - col, r);
    }
  }
}

// out[c] = sum over the n rows of part, in a fixed order: a workgroup takes 32
// columns, 32 threads a column with the rows r, r + 32, ...; their sums are
// added in order.
__global__ __launch_bounds__(1024) void part_sum_kernel(const float* __restrict__ part, float* __restrict__ out, int n,
                                                       int cols) {
  __shared__ float s[32][33];
  const int c = threadIdx.x & 31, r = threadIdx.x >> 5;
  const int col = blockIdx.x * 32 + c;
  float x[4] = {};
  if (col < cols) {
    int k = r;
    // sixteen loads go out together
    for (; k + 480 < n; k += 512) {
      float v[16];
#pragma unroll
      for (int u = 0; u < 16; ++u) v[u] = part[(int64_t)(k + 32 * u) * cols + col];
#pragma unroll
      for (int u = 0; u < 16; ++u) x[u & 3] += v[u];
    }
    for (; k + 96 < n; k += 128)
#pragma unroll
      for (int u = 0; u < 4; ++u) x[u] += part[(int64_t)(k + 32 * u) * cols + col];
    for (; k < n; k += 32) x[0] += part[(int64_t)k * cols + col];
  }
  s[r][c] = (x[0] + x[1]) + (x[2] + x[3]);
  __syncthreads();
  if (r == 0 && col < cols) {
    float sum = 0.0f;
#pragma unroll
    for (int k = 0; k < 32; ++k) sum += s[k][c];
    out[col] = sum;
  }
}

// Threads a row and chunks a thread (one or two: with four the backward's
// sums, the row and its successor no longer fit the registers, nor with two at
// 1024 threads, which have 128 registers each).  One wave a row up to 1024 columns,
// where rows are many: a row's sums then need no barrier.  Few rows, and longer
// ones, take a workgroup each (9479 rows of 6751 into e4m3: 512 threads 131 us,
// 1024 threads 167).
struct RowForm {
  int tpr, nch;           // tpr 0: the long form
};
constexpr int64_t kFewRows = 1024;
RowForm row_form(int64_t rows, int cols, bool fwd) {
  const int chunks = (cols + 7) / 8;
  auto pick = [&](int tpr) { return RowForm{tpr, chunks <= tpr ? 1 : 2}; };
  if (chunks <= 64 || (chunks <= 128 && rows > kFewRows)) return pick(64);
  if (chunks <= 512) return pick(256);
  if (chunks <= 1024) return RowForm{512, 2};
  if (chunks <= 2048 && fwd) return RowForm{1024, 2};
  return RowForm{0, 0};
}

}  // namespace

#define TERRA_ROW_FORM(KERNEL, T, TPR, NCH, THREADS)                                            \
  if (a.cols % 8 == 0) hipLaunchKernelGGL((KERNEL<T, TPR, NCH, false>), grid, dim3(THREADS), 0, st, a); \
  else hipLaunchKernelGGL((KERNEL<T, TPR, NCH, true>), grid, dim3(THREADS), 0, st, a);           \
  break
#define TERRA_ROW_FORMS(KERNEL, T)                              \
  switch (f.tpr + f.nch) {                                      \
    case 65: TERRA_ROW_FORM(KERNEL, T, 64, 1, 256);             \
    case 66: TERRA_ROW_FORM(KERNEL, T, 64, 2, 256);             \
    case 257: TERRA_ROW_FORM(KERNEL, T, 256, 1, 256);           \
    case 258: TERRA_ROW_FORM(KERNEL, T, 256, 2, 256);           \
    case 514: TERRA_ROW_FORM(KERNEL, T, 512, 2, 512);

namespace {

// Workgroups: those that are resident at once on 256 compute units walk the rows.
int row_blocks(int64_t rows, int per, int64_t most) {
  const int64_t b = (rows + per - 1) / per;
  return (int)(b < most ? b : most);
}
int row_blocks(int64_t rows, const RowForm& f, bool bwd) {
  if (f.tpr == 0 || f.tpr >= 512) return row_blocks(rows, 1, 512);
  return row_blocks(rows, f.tpr == 64 ? 4 : 1, 256 * (f.nch == 2 ? (bwd ? 3 : 5) : (bwd ? 5 : 8)));
}

template <typename T>
hipError_t fwd_t(const RmsFwd& a, hipStream_t st) {
  const RowForm f = row_form(a.rows, a.cols, true);
  const dim3 grid(row_blocks(a.rows, f, false));
  if (f.tpr == 0) hipLaunchKernelGGL(rms_fwd_long_kernel<T>, grid, dim3(1024), 0, st, a);
  TERRA_ROW_FORMS(rms_fwd_kernel, T)
    case 1026: TERRA_ROW_FORM(rms_fwd_kernel, T, 1024, 2, 1024);
  }
  return hipGetLastError();
}

template <typename T>
hipError_t bwd_t(const RmsBwd& a, int blocks, hipStream_t st) {
  const RowForm f = row_form(a.rows, a.cols, false);
  const dim3 grid(blocks);
  if (f.tpr == 0) hipLaunchKernelGGL(rms_bwd_long_kernel<T>, grid, dim3(1024), 0, st, a);
  TERRA_ROW_FORMS(rms_bwd_kernel, T)
  }
  return hipGetLastError();
}

}  // namespace
#undef TERRA_ROW_FORMS
#undef TERRA_ROW_FORM

hipError_t launch_part_sum(const float* part, float* out, int n, int cols, hipStream_t st) {
  hipLaunchKernelGGL(part_sum_kernel, dim3((cols + 31) / 32), dim3(1024), 0, st, part, out, n, cols);
  return hipGetLastError();
}

// Workgroups of the backward, each with a row of partial sums; and the most for up to
// so many rows (the form for few rows can have more than that for many).
int rms_bwd_blocks(int64_t rows, int cols) { return row_blocks(rows, row_form(rows, cols, false), true); }
int rms_bwd_most_blocks(int64_t rows, int cols) {
  return std::max(rms_bwd_blocks(rows, cols), rms_bwd_blocks(std::min<int64_t>(rows, kFewRows), cols));
}

hipError_t launch_rms_fwd(int dtype, const RmsFwd& a, hipStream_t st) {
  if (a.rows == 0) return hipSuccess;
  return dtype == 0 ? fwd_t<float>(a, st) : dtype == 1 ? fwd_t<__bf16>(a, st) : fwd_t<_Float16>(a, st);
}

hipError_t launch_rms_bwd(int dtype, RmsBwd a, float* dgain, hipStream_t st) {
  const int blocks = rms_bwd_blocks(a.rows, a.cols);
  const bool alone = dgain != nullptr && blocks == 1;      // one workgroup's sums are the sums
  if (alone) a.part = dgain;
  if (blocks > 0 && (a.dx != nullptr || dgain != nullptr)) {
    const hipError_t e = dtype == 0   ? bwd_t<float>(a, blocks, st)
                         : dtype == 1 ? bwd_t<__bf16>(a, blocks, st)
                                      : bwd_t<_Float16>(a, blocks, st);
    if (e != hipSuccess) return e;
  }
  return dgain == nullptr || alone ? hipSuccess : launch_part_sum(a.part, dgain, blocks, a.cols, st);
}

}  // namespace terra
