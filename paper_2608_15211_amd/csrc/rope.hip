// rope.hip - rotary positions: pairs of a head's channels turned by the angle
// of the token's position, on q and k in one launch.
//
//   (a, b) -> scale (a cos - b sin, a sin + b cos),  angle = position * f_i
// Pair i of an axis holds channels (2i, 2i + 1) of its part of the head, or
// (i, i + half).  The backward is the same with the angles' signs turned.
//
// Angles.  position * f_i loses every digit that counts in float32 at far
// positions, so a frequency comes as turns a position in 64-bit fixed point
// and the product is taken modulo 2^64, which drops the whole turns exactly.  A
// frequency is within 1.5 * 2^-64 turns of its formula (YaRN 2.8 at the usual betas:
// half a unit of its rounding, and the long double steps before it), so an angle is
// off by at most 2.8 |position| 2^-64 turns, and by 2^-32 turns more where the
// product is cut to its upper half: below 6e-10 turns at any 32-bit position,
// besides the float32 steps after it.
//
// What bounds it: HBM, every channel is read and written once.  A workgroup
// takes `tb` tokens: it first works out their cosines and sines, once for all
// heads of q and k, into LDS, then moves units of V pairs, consecutive threads
// along a head.
#include <math.h>

#include <algorithm>

#include "terra_vec.h"
#include "terra_ops.h"

namespace terra {

namespace {

// cos and sin of u / 2^32 turns: the quadrant from the two leading bits (after
// rounding), the rest, |x| <= pi / 4, by the Taylor polynomials to x^9 and x^8
// (next terms below 2e-9 and 3e-8).
__device__ inline float2 cos_sin(uint32_t u) {
  const uint32_t quad = (u + 0x20000000u) >> 30;
  const float x = (float)(int32_t)(u - (quad << 30)) * 1.46291807926715968e-9f;   // 2 pi / 2^32
  const float y = x * x;
  const float s = fmaf(x * y, fmaf(y, fmaf(y, fmaf(y, 2.7557319e-6f, -1.9841270e-4f), 8.3333333e-3f), -1.6666667e-1f), x);
  const float c = fmaf(y, fmaf(y, fmaf(y, fmaf(y, 2.4801587e-5f, -1.3888889e-3f), 4.1666667e-2f), -0.5f), 1.0f);
  const bool swap = quad & 1;
  const float cs = swap ? s : c, sn = swap ? c : s;
  return float2{((quad + 1) & 2) ? -cs : cs, (quad & 2) ? -sn : sn};
}

template <typename T, int V>
struct Vec {
  T v[V];
};

// Threads a workgroup, and the LDS floats its angles may take.
constexpr int kRopeThreads = 256;
constexpr int kRopeAngles = 4096;

// V pairs from the first one's channels: in the half layout the second of a pair
// is `half` channels on, in the interleaved one the next.
template <typename T, int V, bool HALF>
__device__ inline void turn_pairs(const T* in, T* out, int half, const float2* cs) {
  T x[V], y[V], p[2 * V];
  if constexpr (HALF) {
    __builtin_memcpy(x, in, sizeof(x));
    __builtin_memcpy(y, in + half, sizeof(y));
  } else {
    __builtin_memcpy(p, in, sizeof(p));
  }
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const float2 c = cs[i];
    const float xf = to_float<T>(HALF ? x[i] : p[2 * i]), yf = to_float<T>(HALF ? y[i] : p[2 * i + 1]);
    const T u = from_float<T>(fmaf(xf, c.x, -yf * c.y)), v = from_float<T>(fmaf(xf, c.y, yf * c.x));
    if constexpr (HALF) { x[i] = u; y[i] = v; }
    else { p[2 * i] = u; p[2 * i + 1] = v; }
  }
  if constexpr (HALF) {
    __builtin_memcpy(out, x, sizeof(x));
    __builtin_memcpy(out + half, y, sizeof(y));
  } else {
    __builtin_memcpy(out, p, sizeof(p));
  }
}
// Up to V pairs, `left` of them there: all at once, or by halves (138240 tokens of
// 2 x 24 heads of 32, 13 pairs, bf16: 443 us, 370 interleaved; pair by pair 724 and 621).
template <typename T, int V, bool HALF>
__device__ inline void turn_some(const T* in, T* out, int half, const float2* cs, int left) {
  if (left >= V) return turn_pairs<T, V, HALF>(in, out, half, cs);
  if constexpr (V > 1) {
    constexpr int W = V / 2, C = HALF ? W : 2 * W;
    if (left >= W) {
      turn_pairs<T, W, HALF>(in, out, half, cs);
      in += C; out += C; cs += W; left -= W;
    }
    if (left > 0) turn_some<T, W, HALF>(in, out, half, cs, left);
  }
}
// Fewer than 2 V channels copied, by halves.
template <typename T, int V>
__device__ inline void copy_some(const T* in, T* out, int left) {
  if (left >= V) {
    T x[V];
    __builtin_memcpy(x, in, sizeof(x));
    __builtin_memcpy(out, x, sizeof(x));
    in += V; out += V; left -= V;
  }
  if constexpr (V > 1)
    if (left > 0) copy_some<T, V / 2>(in, out, left);
}

template <typename T, int V, bool HALF>
__global__ __launch_bounds__(kRopeThreads) void rope_kernel(RopeArgs a) {
  extern __shared__ float2 angles[];       // [tb][pairs]
  const int64_t blocks = (a.tokens + a.tb - 1) / a.tb;
  for (int64_t blk = blockIdx.x; blk < blocks; blk += gridDim.x) {
    if (blk != blockIdx.x) __syncthreads();     // the angles of the last tokens are used
    const int64_t tok0 = blk * a.tb;
    const int ntok = (int)min((int64_t)a.tb, a.tokens - tok0);
    for (int idx = threadIdx.x; idx < ntok * a.pairs; idx += kRopeThreads) {
      const int t = fast_div(idx, a.pairs, a.rpairs), p = idx - t * a.pairs;
      const int axis = p >= a.half ? 1 : 0;
      const int64_t tok = tok0 + t;
      int64_t pos;
      if (a.pos != nullptr) {
        pos = a.pos[tok * a.axes + axis];
      } else {
        const uint32_t cell = (uint32_t)(tok % (int64_t)a.grid_hw);
        pos = a.axes == 1 ? cell : axis == 0 ? cell / (uint32_t)a.grid_w : cell % (uint32_t)a.grid_w;
      }
      float2 cs = cos_sin((uint32_t)(((uint64_t)pos * a.turns[p - axis * a.half]) >> 32));
      angles[idx] = float2{cs.x * a.scale, cs.y * a.sin_scale};
    }
    __syncthreads();

    // units of a token: q's heads, then k's; a head's turned units of V pairs,
    // then the copied ones of 2 V channels
    const int total = ntok * a.units;
    for (int idx = threadIdx.x; idx < total; idx += kRopeThreads) {
      const int t = fast_div(idx, a.units, a.runits);
      const int rem = idx - t * a.units;
      int head = fast_div(rem, a.uph, a.ruph);
      const int u = rem - head * a.uph;
      const bool second = head >= a.side[0].heads;
      const RopeSide& s = second ? a.side[1] : a.side[0];
      if (second) head -= a.side[0].heads;
      const T* in = (const T*)s.in + (tok0 + t) * s.in_t + head * s.in_h;
      T* out = (T*)s.out + (tok0 + t) * s.out_t + head * s.out_h;
      if (u < a.turned) {
        // pairs [i, i + V) of an axis, as many as there are
        const int axis = u >= a.upa ? 1 : 0;
        const int i = (u - axis * a.upa) * V, left = a.half - i;
        const float2* cs = angles + t * a.pairs + axis * a.half + i;
        // channels of the first pair
        const int lo = 2 * axis * a.half + (HALF ? i : 2 * i);
        turn_some<T, V, HALF>(in + lo, out + lo, a.half, cs, left);
      } else {
        // copied channels; the last unit ends with the head and may repeat some
        const int c0 = 2 * a.pairs + (u - a.turned) * 2 * V;
        if (a.hd - 2 * a.pairs >= 2 * V) {
          const int c = min(c0, a.hd - 2 * V);
          Vec<T, 2 * V> x;
          __builtin_memcpy(&x, in + c, sizeof(x));
          __builtin_memcpy(out + c, &x, sizeof(x));
        } else {
          copy_some<T, V>(in + c0, out + c0, a.hd - c0);
        }
      }
    }
  }
}

template <typename T, int V>
hipError_t rope_form(const RopeArgs& a, bool half, hipStream_t st) {
  const dim3 grid((unsigned)std::min<int64_t>((a.tokens + a.tb - 1) / a.tb, 1 << 20));
  const size_t lds = (size_t)a.tb * a.pairs * sizeof(float2);
  if (half) hipLaunchKernelGGL((rope_kernel<T, V, true>), grid, dim3(kRopeThreads), lds, st, a);
  else hipLaunchKernelGGL((rope_kernel<T, V, false>), grid, dim3(kRopeThreads), lds, st, a);
  return hipGetLastError();
}

template <typename T>
hipError_t rope_t(const RopeArgs& a, int v, bool half, hipStream_t st) {
  return v == 8   ? rope_form<T, 8>(a, half, st)
         : v == 4 ? rope_form<T, 4>(a, half, st)
         : v == 2 ? rope_form<T, 2>(a, half, st)
                  : rope_form<T, 1>(a, half, st);
}

}  // namespace

// turns[i] = f_i / (2 pi) in units of 2^-64, for the pairs of one axis.
void rope_turns(double base, int scaling, double factor, double orig_len, double beta_fast, double beta_slow, int part,
                uint64_t* turns) {
  const long double two_pi = 6.283185307179586476925286766559005768L;
  const long double b = scaling == 2 ? base * powl(factor, (long double)part / (part - 2)) : base;
  for (int i = 0; i < part / 2; ++i) {
    long double f = powl(b, -2.0L * i / part) / two_pi;
    if (scaling == 1) f /= factor;
    if (scaling == 3) {
      long double keep = (orig_len * f - beta_slow) / (beta_fast - beta_slow);
      keep = keep < 0 ? 0 : keep > 1 ? 1 : keep;
      f *= keep + (1 - keep) / factor;
    }
    turns[i] = (uint64_t)rintl(ldexpl(f, 64));
  }
}

hipError_t launch_rope(int dtype, RopeArgs a, bool half, hipStream_t st) {
  if (a.tokens == 0) return hipSuccess;
  // pairs a unit: 8 (16-byte accesses of 16-bit types), fewer where an axis has
  // fewer or half as many leave none over; what is left goes by fours, twos and ones (26 pairs
  // of 24 heads: 13.9 us against 15.8 in units of two; 6 pairs: 11.8 in units of
  // four, 9 in units of two)
  int v = 8;
  while (v > a.half || (v > 2 && a.half % v != 0 && a.half % (v / 2) == 0)) v /= 2;
  const bool in_place = a.side[0].in == a.side[0].out && (a.side[1].heads == 0 || a.side[1].in == a.side[1].out);
  const bool copy = a.hd > 2 * a.pairs && !in_place;
  a.upa = (a.half + v - 1) / v;
  a.turned = a.axes * a.upa;
  a.uph = a.turned + (copy ? (a.hd - 2 * a.pairs + 2 * v - 1) / (2 * v) : 0);
  a.units = a.uph * (a.side[0].heads + a.side[1].heads);
  // tokens a workgroup: about two units a thread (138240 tokens of 2 x 24 heads of
  // 32, bf16: 164 us, with six 178; 31401 of 15 heads of 64 29.6 and 32.7), while
  // the angles fit, and fewer where that would leave compute units idle
  int64_t tb = (2 * kRopeThreads + a.units - 1) / a.units;
  tb = std::min<int64_t>(tb, std::max(1, kRopeAngles / a.pairs));
  tb = std::min<int64_t>(tb, std::max<int64_t>(1, a.tokens / 1024));
  a.tb = (int)tb;
  a.rpairs = 1.0f / (float)a.pairs;
  a.runits = 1.0f / (float)a.units;
  a.ruph = 1.0f / (float)a.uph;
  return dtype == 0 ? rope_t<float>(a, v, half, st) : dtype == 1 ? rope_t<__bf16>(a, v, half, st) : rope_t<_Float16>(a, v, half, st);
}

}  // namespace terra
