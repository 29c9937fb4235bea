// terra_vec.h - chunks of eight elements between memory and float32 registers,
// for tensors of any row length, stride and alignment.
//
// A chunk inside its row moves as one 16-byte access (32 bytes of float32,
// 8 of e4m3) whatever its address: global accesses need the element's
// alignment only.  The last chunk of a row whose length is no multiple of
// eight moves element by element and never touches what lies behind the row.
#pragma once

#include <string.h>

#include "terra_common.h"

namespace terra {

constexpr float kE4m3Max = 448.0f;

template <typename T>
struct Chunk {
  T v[8];
};

// A chunk as it is in memory: elements [0, n) of it, the rest zero.  RAG: n may be
// anything; else it is at least 8 or the chunk lies outside the row.
template <bool RAG, typename T>
__device__ inline Chunk<T> fetch8(const T* p, int n) {
  Chunk<T> c;
  if (n >= 8) {
    __builtin_memcpy(&c, p, sizeof(c));
  } else {
    __builtin_memset(&c, 0, sizeof(c));
    if (RAG && n > 0) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < n) c.v[i] = p[i];
    }
  }
  return c;
}
template <typename T>
__device__ inline void widen8(const Chunk<T>& c, float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = to_float<T>(c.v[i]);
}
// Where n >= 8 or the chunk lies outside, or RAG.
template <bool RAG, typename T>
__device__ inline void put8(T* p, int n, const float (&f)[8]);

// Elements [0, n) of a chunk (n >= 8: all), the rest zero.
template <typename T>
__device__ inline void load8(const T* p, int n, float (&f)[8]) {
  if (n >= 8) {
    Chunk<T> c;
    __builtin_memcpy(&c, p, sizeof(c));
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = to_float<T>(c.v[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = i < n ? to_float<T>(p[i]) : 0.0f;
  }
}

template <typename T>
__device__ inline void store8(T* p, int n, const float (&f)[8]) {
  if (n >= 8) {
    Chunk<T> c;
#pragma unroll
    for (int i = 0; i < 8; ++i) c.v[i] = from_float<T>(f[i]);
    __builtin_memcpy(p, &c, sizeof(c));
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = from_float<T>(f[i]);
  }
}

template <bool RAG, typename T>
__device__ inline void put8(T* p, int n, const float (&f)[8]) {
  if (RAG) store8(p, n, f);
  else if (n >= 8) store8(p, 8, f);
}

// Eight floats to e4m3, rounded to nearest even; |f| is at most 448 but for
// float32's own rounding.
__device__ inline void store8_e4m3(uint8_t* p, int n, const float (&f)[8]) {
  int w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    w[i] = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * i], f[4 * i + 1], 0, false);
    w[i] = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * i + 2], f[4 * i + 3], w[i], true);
  }
  if (n >= 8) {
    __builtin_memcpy(p, w, 8);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = (uint8_t)((uint32_t)w[i >> 2] >> (8 * (i & 3)));
  }
}

}  // namespace terra
