// Pieces shared by the kernels that work on rows in memory (rmsnorm.hip, rotary.hip): V consecutive elements of a row as
// floats, sums and maxima over the threads that share a row, and the refusals of entry points that take no context.
#pragma once

#include <string>

#include "common.h"

namespace reslim {

// 16 and 8 bytes from any address: one access of gfx950 whether or not it is a multiple of its size
typedef __attribute__((ext_vector_type(4), aligned(1))) uint32_t u32x4_row;
typedef __attribute__((ext_vector_type(2), aligned(1))) uint32_t u32x2_row;
typedef uint32_t __attribute__((aligned(1))) u32_row;
typedef __attribute__((ext_vector_type(4), aligned(4))) float f32x4_row;

struct e4m3_t { uint8_t bits; };      // sign, 4 bits of exponent (bias 7), 3 of mantissa; largest 448, no infinities
constexpr float kE4m3Max = 448.0f;

// four floats to e4m3, to nearest, ties to even
__device__ __forceinline__ uint32_t pack_e4m3x4(float a, float b, float c, float d) {
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true));
}

// V consecutive elements, from any element on
template <class T, int V> struct Piece;
template <int V> struct Piece<float, V> {
  static __device__ __forceinline__ void load(const float *p, float (&v)[V]) {
    if constexpr (V % 4 == 0) {
#pragma unroll
      for (int i = 0; i < V; i += 4) {
        const f32x4_row f = *reinterpret_cast<const f32x4_row *>(p + i);
        v[i] = f[0]; v[i + 1] = f[1]; v[i + 2] = f[2]; v[i + 3] = f[3];
      }
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] = p[i];
    }
  }
  static __device__ __forceinline__ void store(float *p, const float (&v)[V]) {
    if constexpr (V % 4 == 0) {
#pragma unroll
      for (int i = 0; i < V; i += 4) *reinterpret_cast<f32x4_row *>(p + i) = f32x4_row{v[i], v[i + 1], v[i + 2], v[i + 3]};
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) p[i] = v[i];
    }
  }
};
template <int V> struct Piece<bf16_t, V> {
  static __device__ __forceinline__ void load(const bf16_t *p, float (&v)[V]) {
    uint32_t w[(V + 1) / 2];
    if constexpr (V == 8) {
      const u32x4_row r = *reinterpret_cast<const u32x4_row *>(p);
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = r[i];
    } else if constexpr (V == 4) {
      const u32x2_row r = *reinterpret_cast<const u32x2_row *>(p);
      w[0] = r[0]; w[1] = r[1];
    } else if constexpr (V == 2) {
      w[0] = *reinterpret_cast<const u32_row *>(p);
    } else {
      w[0] = *p;
    }
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = __uint_as_float(i % 2 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
  }
  static __device__ __forceinline__ void store(bf16_t *p, const float (&v)[V]) {
    if constexpr (V == 8) {
      *reinterpret_cast<u32x4_row *>(p) = u32x4_row{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
    } else if constexpr (V == 4) {
      *reinterpret_cast<u32x2_row *>(p) = u32x2_row{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
    } else if constexpr (V == 2) {
      *reinterpret_cast<u32_row *>(p) = pack_bf16x2(v[0], v[1]);
    } else {
      *p = f32_to_bf16(v[0]);
    }
  }
};
template <int V> struct Piece<e4m3_t, V> {
  static __device__ __forceinline__ void store(e4m3_t *p, const float (&v)[V]) {
    if constexpr (V == 8) {
      *reinterpret_cast<u32x2_row *>(p) = u32x2_row{pack_e4m3x4(v[0], v[1], v[2], v[3]), pack_e4m3x4(v[4], v[5], v[6], v[7])};
    } else if constexpr (V == 4) {
      *reinterpret_cast<u32_row *>(p) = pack_e4m3x4(v[0], v[1], v[2], v[3]);
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) p[i].bits = static_cast<uint8_t>(pack_e4m3x4(v[i], 0.f, 0.f, 0.f) & 0xff);
    }
  }
};

// The same elements as they lie in memory, to be held until they are used.
template <class T, int V> struct Held {
  static constexpr int kWords = (V * static_cast<int>(sizeof(T)) + 3) / 4;
  uint32_t w[kWords];
  __device__ __forceinline__ void load(const T *p) {
    if constexpr (kWords % 4 == 0) {
#pragma unroll
      for (int i = 0; i < kWords; i += 4) {
        const u32x4_row r = *reinterpret_cast<const u32x4_row *>(reinterpret_cast<const uint32_t *>(p) + i);
        w[i] = r[0]; w[i + 1] = r[1]; w[i + 2] = r[2]; w[i + 3] = r[3];
      }
    } else if constexpr (kWords == 2) {
      const u32x2_row r = *reinterpret_cast<const u32x2_row *>(p);
      w[0] = r[0]; w[1] = r[1];
    }
    static_assert(kWords % 2 == 0, "whole pieces of 8 or 16 bytes");
  }
  __device__ __forceinline__ void load_some(const T *p, int n) {      // the first n
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = 0;
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i < n) {
        if constexpr (sizeof(T) == 4) w[i] = reinterpret_cast<const uint32_t *>(p)[i];
        else w[i / 2] |= static_cast<uint32_t>(reinterpret_cast<const uint16_t *>(p)[i]) << (i % 2 * 16);
      }
  }
  __device__ __forceinline__ float operator[](int i) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
    else return __uint_as_float(i % 2 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
  }
};

// ... and the first n of V elements, zeros behind them
template <class T, int V>
__device__ __forceinline__ void load_some(const T *p, int n, float (&v)[V]) {
#pragma unroll
  for (int i = 0; i < V; ++i) {
    float f[1] = {0.f};
    if (i < n) Piece<T, 1>::load(p + i, f);
    v[i] = f[0];
  }
}
template <class T, int V>
__device__ __forceinline__ void store_some(T *p, int n, const float (&v)[V]) {
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const float f[1] = {v[i]};
    if (i < n) Piece<T, 1>::store(p + i, f);
  }
}

// Sum (or maximum) over the NT threads that share a row, the same value in all of them.  box: NT / 64 floats of LDS that nothing
// else uses until every thread is past the call after next (two boxes taken in turn).
template <int NT, bool MAX>
__device__ __forceinline__ float row_all(float s, float *box) {
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    const float o = __shfl_xor(s, m);
    s = MAX ? fmaxf(s, o) : s + o;
  }
  if constexpr (NT > 64) {
    if ((threadIdx.x & 63) == 0) box[threadIdx.x >> 6] = s;
    __syncthreads();
    s = box[0];
#pragma unroll
    for (int w = 1; w < NT / 64; ++w) s = MAX ? fmaxf(s, box[w]) : s + box[w];
  }
  return s;
}

// Two sums at once, over one barrier; box: 2 NT / 64 floats
template <int NT>
__device__ __forceinline__ void row_sum2(float &a, float &b, float *box) {
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    a += __shfl_xor(a, m);
    b += __shfl_xor(b, m);
  }
  if constexpr (NT > 64) {
    constexpr int W = NT / 64;
    if ((threadIdx.x & 63) == 0) {
      box[threadIdx.x >> 6] = a;
      box[W + (threadIdx.x >> 6)] = b;
    }
    __syncthreads();
    a = box[0];
#pragma unroll
    for (int w = 1; w < W; ++w) a += box[w];
    if constexpr (W == 16) __builtin_amdgcn_sched_barrier(0);      // sixteen values at a time
    b = box[W];
#pragma unroll
    for (int w = 1; w < W; ++w) b += box[W + w];
  }
}

// An entry point without a context refuses: the text goes to reslim_last_error(NULL).  Throws nothing.
inline int refuse(int code, const char *fn, const char *why) noexcept {
  try {
    set_thread_error(std::string(fn) + ": " + why);
  } catch (...) {
  }
  return code;
}
inline int refuse_hip(const char *fn, hipError_t e) noexcept { return refuse(RESLIM_EHIP, fn, hipGetErrorString(e)); }

// Work-groups of one launch: a launch holds fewer than 2^32 threads.
constexpr int64_t most_groups(int threads) { return (int64_t{1} << 31) / threads; }

inline bool aligned(const void *p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }
inline size_t type_bytes(int dtype) { return dtype == RESLIM_F32 ? 4 : dtype == RESLIM_BF16 ? 2 : 1; }

}  // namespace reslim
