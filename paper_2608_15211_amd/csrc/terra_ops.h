// terra_ops.h - argument blocks of the operators around the attention
// (norm.hip, linear.hip, rope.hip), filled by the C ABI (abi.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace terra {

struct RmsFwd {
  const void *x, *res;
  const float* gain;
  void *z, *y;
  uint8_t* q;
  float *q_scale, *rstd;
  int64_t rows, x_ld, res_ld, z_ld, y_ld, q_ld;
  int cols;
  float eps;
};

struct RmsBwd {
  const void *dy, *z, *dz;
  const float *rstd, *gain;
  void* dx;
  float* part;             // partial sums of dgain, a row for each workgroup
  int64_t rows, dy_ld, z_ld, dz_ld, dx_ld;
  int cols;
};

// out[c] = sum over the n rows of part ([n][cols]), in a fixed order.
hipError_t launch_part_sum(const float* part, float* out, int n, int cols, hipStream_t st);

int rms_bwd_blocks(int64_t rows, int cols);
int rms_bwd_most_blocks(int64_t rows, int cols);
hipError_t launch_rms_fwd(int dtype, const RmsFwd& a, hipStream_t st);
hipError_t launch_rms_bwd(int dtype, RmsBwd a, float* dgain, hipStream_t st);

constexpr int kRopePairs = 128;    // of one head, at most

struct RopeSide {
  const void* in;
  void* out;
  int heads;
  int64_t in_t, in_h, out_t, out_h;     // token and head strides, elements
};

struct RopeArgs {
  RopeSide side[2];
  int64_t tokens;
  const int32_t* pos;      // [tokens][axes], or null: the token's place on the grid
  int axes, half, pairs;   // pairs of one axis, of a head
  int hd;
  uint32_t grid_w, grid_hw;
  float scale, sin_scale;  // factors on cosine and sine
  // set by launch_rope: tokens a workgroup, units of a token and of a head,
  // how many of these turn, of an axis, and the reciprocals fast_div starts from
  int tb, units, uph, turned, upa;
  float rpairs, runits, ruph;
  uint64_t turns[kRopePairs];
};

void rope_turns(double base, int scaling, double factor, double orig_len, double beta_fast, double beta_slow, int part,
                uint64_t* turns);
hipError_t launch_rope(int dtype, RopeArgs a, bool half, hipStream_t st);

// Element types of the linear layer's operands; kE4m3's outputs are 16-bit.
enum { kF32 = 0, kBf16 = 1, kF16 = 2, kE4m3 = 3 };
enum { kActNone = 0, kActRelu = 1, kActGelu = 2, kActSilu = 3 };

struct LinFwd {
  const void *x, *w;                    // [M][K], [N][K]; strides in elements
  const float *x_scale, *w_scale;       // e4m3: of each row
  const float* bias;
  const void* res;
  void *y, *pre;
  int64_t M, x_ld, w_ld, y_ld, res_ld, pre_ld;
  int N, K, act;
};

struct LinBwd {
  const void *dy, *x, *w, *pre;
  void *dx, *dw;
  float* db;
  int64_t M, dy_ld, x_ld, w_ld, pre_ld, dx_ld, dw_ld;
  int N, K, act;
  bool dw_f32;
};

int lin_form(int64_t M, int N, int K, int dtype, bool aligned);
int lin_few_waves(int64_t M, int N, int K, int dtype);
int lin_wgrad_form(int64_t M, int N, int K, bool aligned);
size_t lin_fwd_workspace(int64_t M, int N, int K, int dtype);
size_t lin_bwd_workspace(int64_t M, int N, int K);
hipError_t launch_lin_fwd(int dtype, int out, const LinFwd& a, void* ws, hipStream_t st);
hipError_t launch_lin_bwd(int dtype, const LinBwd& a, void* ws, hipStream_t st);

}  // namespace terra
