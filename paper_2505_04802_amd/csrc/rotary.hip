// Rotary positions: pair j of a head's first `rot` features turns by the angle position * frequency[j],
//   (a, b) -> amplitude (a cos - b sin, a sin + b cos),        gradient: the transpose, the same turn backwards,
// pairs (2j, 2j + 1) (interleaved) or (j, j + rot / 2) (halves); with two axes the first half of the pairs turns by the first
// coordinate and the second half by the second.
//
// Every rotated head is read and written once, and memory bounds it; what could cost more is the angle.  It is formed in
// 64 bits (at position 10^6 a 32-bit product of position and frequency is off by 0.06 radians), reduced to a fraction of a turn there, and
// its sine and cosine are taken in 32.  A thread takes one 16-byte piece of a head (two where the pairs are halves) at the same
// place in several heads of a token, so that an angle serves them all.  161,408 tokens x 32 heads of 64 (bf16, two axes) take 242 us, 5.4 TB/s;
// 16 tokens x 40 heads of 128 4.5 us, the latencies of position, frequency, angle and data in a row.
#include <algorithm>
#include <cmath>

#include "rows_common.h"

namespace reslim {

struct RotaryArgs {
  const void *x;
  void *out;
  const int32_t *positions;      // [axes, period]
  const double *freq;            // [rot / 2]
  int64_t tokens, x_stride, out_stride, period;      // strides: elements from token to token
  int64_t first;                 // number of the first token
  int heads, dh, rot, axes;
  int pieces, lanes;             // of a head: threads over it; threads over the heads
  int copy;                      // write the features behind `rot` too
  float amplitude, sign;
};

// sin and cos of 2 pi f, |f| <= 1/2
__device__ __forceinline__ void turn(double angle, float amplitude, float sign, float &c, float &s) {
  const double t = angle * 0.15915494309189533576888;
  const float f = static_cast<float>(t - rint(t));
  float sn, cs;
  sincospif(2.0f * f, &sn, &cs);
  c = amplitude * cs;
  s = amplitude * sign * sn;
}

// V: features of a piece; HALVES: pairs (j, j + rot / 2), two pieces a thread.  Threads behind the turning pieces copy, on the same path (the
// other one would cost every wave the latency of both): 25,986 x 20 heads of 128, half of each turning, 81 us with a path of their own.
template <class T, int V, bool HALVES>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryArgs a) {
  constexpr int NP = HALVES ? V : V / 2;       // pairs of a thread
  const int per_token = a.pieces * a.lanes;
  const int tpb = per_token < 256 ? 256 / per_token : 1;      // tokens of a work-group
  const int slot = threadIdx.x / per_token;
  const int64_t token = static_cast<int64_t>(blockIdx.x) * tpb + slot;
  if (slot >= tpb || token >= a.tokens) return;
  const int within = threadIdx.x % per_token;
  const int turning = a.rot / 2 / NP;
  const int64_t at = (a.first + token) % a.period;
  const T *x = static_cast<const T *>(a.x) + token * a.x_stride;
  T *o = static_cast<T *>(a.out) + token * a.out_stride;
  for (int u = within; u < per_token; u += 256) {      // more than one round only where a head has more than 256 pieces
    const int piece = u % a.pieces, lane = u / a.pieces;
    const bool turns = piece < turning;
    float c[NP], s[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int j = turns ? piece * NP + i : 0;
      const int axis = 2 * j * a.axes / a.rot;           // 0, or 1 in the second half of the pairs
      turn(static_cast<double>(a.positions[axis * a.period + at]) * a.freq[j], a.amplitude, a.sign, c[i], s[i]);
    }
    const int k0 = turns ? piece * (HALVES ? V : 2 * NP) : a.rot + (piece - turning) * (HALVES ? 2 * V : V);
    const int k1 = turns ? k0 + a.rot / 2 : k0 + V;
    const bool two = HALVES && k1 < a.dh;                // the last copied piece may be single
    constexpr int G = 4;                       // heads whose loads are in flight together
    for (int h0 = lane; h0 < a.heads; h0 += G * a.lanes) {
      float p[G][V], q[G][HALVES ? V : 1];
#pragma unroll
      for (int g = 0; g < G; ++g) {
        const int h = h0 + g * a.lanes;
        if (h < a.heads) {
          Piece<T, V>::load(x + h * a.dh + k0, p[g]);
          if constexpr (HALVES) {
            if (two) Piece<T, V>::load(x + h * a.dh + k1, q[g]);
          }
        }
      }
#pragma unroll
      for (int g = 0; g < G; ++g) {
        const int h = h0 + g * a.lanes;
        if (h >= a.heads) break;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
          float &f0 = HALVES ? p[g][i] : p[g][2 * i], &f1 = HALVES ? q[g][HALVES ? i : 0] : p[g][HALVES ? 0 : 2 * i + 1];
          const float u0 = f0, u1 = f1;
          f0 = turns ? u0 * c[i] - u1 * s[i] : u0;
          f1 = turns ? u0 * s[i] + u1 * c[i] : u1;
        }
        Piece<T, V>::store(o + h * a.dh + k0, p[g]);
        if constexpr (HALVES) {
          if (two) Piece<T, V>::store(o + h * a.dh + k1, q[g]);
        }
      }
    }
  }
}

template <class T, int V, bool HALVES>
static hipError_t launch_rotary_v(RotaryArgs a, hipStream_t st) {
  const int np = HALVES ? V : V / 2, copied = HALVES ? 2 * V : V;
  a.pieces = a.rot / 2 / np + (a.copy ? (a.dh - a.rot + copied - 1) / copied : 0);
  // An angle serves the heads that a thread walks through; threads over the heads are added while the launch leaves the
  // chip without eight waves on a compute unit, down to one head a thread.
  int lanes = (a.heads + 7) / 8;
  while (lanes < a.heads && a.tokens * a.pieces * lanes < 256LL * 8 * 64) lanes *= 2;
  const int most = a.pieces < 256 ? 256 / a.pieces : 1;
  a.lanes = lanes < a.heads ? lanes : a.heads;
  if (a.lanes > most) a.lanes = most;
  const int per_token = a.pieces * a.lanes, tpb = per_token < 256 ? 256 / per_token : 1;
  for (int64_t left = a.tokens; left > 0;) {
    a.tokens = std::min(left, most_groups(256) * tpb);
    rotary_kernel<T, V, HALVES><<<dim3(static_cast<unsigned>((a.tokens + tpb - 1) / tpb)), dim3(256), 0, st>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    a.x = static_cast<const T *>(a.x) + a.tokens * a.x_stride;
    a.out = static_cast<T *>(a.out) + a.tokens * a.out_stride;
    a.first += a.tokens;
    left -= a.tokens;
  }
  return hipSuccess;
}

// The widest pieces, up to 16 bytes, that neither the turning part (either half of it where pairs are halves) nor the head ends inside.  With single elements 25,986 x 20 heads of 96, 24 of them turning as halves, took 117 us.
// In place, where the features behind the turning part are not touched, too: pieces of 16 bytes from any address are no faster in heads of 70 or 130 (25,986 x 20 heads of
// 70, 64 of them turning, 28.2 us; with the pieces of two that divide the six others 27.4).
template <class T, bool HALVES, int V>
static hipError_t launch_rotary(const RotaryArgs &a, hipStream_t st) {
  if constexpr (V > (HALVES ? 1 : 2)) {
    if ((a.dh - a.rot) % V || a.rot % (HALVES ? 2 * V : V)) return launch_rotary<T, HALVES, V / 2>(a, st);
  }
  return launch_rotary_v<T, V, HALVES>(a, st);
}

static int rotary_impl(const char *fn, const void *x, void *out, const int32_t *positions, const double *freq, int64_t tokens, int64_t x_stride, int64_t out_stride,
                       int64_t period, int32_t heads, int32_t dh, int32_t rot, int32_t axes, int32_t layout, float amplitude, int32_t dtype, float sign, void *hip_stream) {
  if (dtype != RESLIM_F32 && dtype != RESLIM_BF16) return refuse(RESLIM_EINVAL, fn, "dtype must be RESLIM_F32 or RESLIM_BF16");
  if (layout != RESLIM_ROTARY_INTERLEAVED && layout != RESLIM_ROTARY_HALVES) return refuse(RESLIM_EINVAL, fn, "unknown layout");
  if (axes != 1 && axes != 2) return refuse(RESLIM_EINVAL, fn, "axes must be 1 or 2");
  if (tokens < 0 || heads < 1 || heads > 65536 || dh < 2 || dh > 1024 || dh % 2 || rot < 2 || rot > dh || rot % (2 * axes) || (tokens > 0 && period < 1))
    return refuse(RESLIM_ESHAPE, fn, "need tokens >= 0, period >= 1, 1 <= heads <= 65536, an even head of 2 to 1024 features and 2 <= rot <= dh, a multiple of 2 axes");
  if (x_stride < static_cast<int64_t>(heads) * dh || out_stride < static_cast<int64_t>(heads) * dh) return refuse(RESLIM_ESHAPE, fn, "a token's stride is shorter than its rotated heads");
  if (!(std::fabs(amplitude) <= 3.402823466e+38f)) return refuse(RESLIM_EINVAL, fn, "amplitude must be finite");
  if (tokens > 0 && (!x || !out || !positions || !freq)) return refuse(RESLIM_EINVAL, fn, "null buffer");
  const size_t es = type_bytes(dtype);
  const bool words = dtype == RESLIM_BF16 && layout == RESLIM_ROTARY_INTERLEAVED;      // pairs of bf16 move as one word
  if (!aligned(x, es) || !aligned(out, es) || !aligned(positions, 4) || !aligned(freq, 8)) return refuse(RESLIM_EINVAL, fn, "a buffer is not aligned to its elements");
  if (words && (!aligned(x, 4) || !aligned(out, 4) || x_stride % 2 || out_stride % 2))
    return refuse(RESLIM_EINVAL, fn, "interleaved bf16 pairs must start on 4 bytes");
  if (tokens > 0 && x == out && x_stride != out_stride) return refuse(RESLIM_EINVAL, fn, "in place the strides must be the same");
  if (tokens == 0) return RESLIM_OK;
  RotaryArgs a = {x, out, positions, freq, tokens, x_stride, out_stride, period, 0, heads, dh, rot, axes, 0, 0, x != out, amplitude, sign};
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  const bool halves = layout == RESLIM_ROTARY_HALVES;
  const hipError_t e = dtype == RESLIM_BF16 ? (halves ? launch_rotary<bf16_t, true, 8>(a, st) : launch_rotary<bf16_t, false, 8>(a, st))
                                            : (halves ? launch_rotary<float, true, 4>(a, st) : launch_rotary<float, false, 4>(a, st));
  return e == hipSuccess ? RESLIM_OK : refuse_hip(fn, e);
}

}  // namespace reslim

using namespace reslim;

extern "C" int reslim_rotary_fwd(const void *x, void *out, const int32_t *positions, const double *freq, int64_t tokens, int64_t x_stride, int64_t out_stride,
                                 int64_t period, int32_t heads, int32_t dh, int32_t rot, int32_t axes, int32_t layout, float amplitude, int32_t dtype, void *hip_stream) {
  return rotary_impl("reslim_rotary_fwd", x, out, positions, freq, tokens, x_stride, out_stride, period, heads, dh, rot, axes, layout, amplitude, dtype, 1.0f, hip_stream);
}

extern "C" int reslim_rotary_bwd(const void *d_out, void *d_x, const int32_t *positions, const double *freq, int64_t tokens, int64_t d_out_stride, int64_t d_x_stride,
                                 int64_t period, int32_t heads, int32_t dh, int32_t rot, int32_t axes, int32_t layout, float amplitude, int32_t dtype, void *hip_stream) {
  return rotary_impl("reslim_rotary_bwd", d_out, d_x, positions, freq, tokens, d_out_stride, d_x_stride, period, heads, dh, rot, axes, layout, amplitude, dtype, -1.0f, hip_stream);
}

// HOST arithmetic in 64 bits.
extern "C" int reslim_rotary_frequencies(int32_t rot, int32_t axes, double base, int32_t scaling, double factor, double original_length, double *freq, float *amplitude) {
  const char *fn = "reslim_rotary_frequencies";
  if (!freq || !amplitude) return refuse(RESLIM_EINVAL, fn, "null argument");
  if ((axes != 1 && axes != 2) || rot < 2 || rot > 1024 || rot % (2 * axes)) return refuse(RESLIM_ESHAPE, fn, "need 1 or 2 axes and 2 <= rot <= 1024, a multiple of 2 axes");
  if (scaling < RESLIM_ROTARY_PLAIN || scaling > RESLIM_ROTARY_BY_PARTS) return refuse(RESLIM_EINVAL, fn, "unknown scaling");
  if (!(base > 1.0) || !std::isfinite(base)) return refuse(RESLIM_EINVAL, fn, "base must be finite and above 1");
  if (scaling != RESLIM_ROTARY_PLAIN && (!(factor >= 1.0) || !std::isfinite(factor))) return refuse(RESLIM_EINVAL, fn, "factor must be finite and at least 1");
  if (scaling == RESLIM_ROTARY_BY_PARTS && (!(original_length >= 1.0) || !std::isfinite(original_length)))
    return refuse(RESLIM_EINVAL, fn, "original_length must be finite and at least 1");
  const int d = rot / axes, n = d / 2;
  if (scaling == RESLIM_ROTARY_BASE && d > 2) base *= std::pow(factor, static_cast<double>(d) / (d - 2));
  for (int j = 0; j < n; ++j) {
    double f = std::pow(base, -2.0 * j / d);
    if (scaling == RESLIM_ROTARY_LINEAR) f /= factor;
    if (scaling == RESLIM_ROTARY_BY_PARTS) {
      const double turns = original_length * f / 6.283185307179586476925;      // over the original context
      double keep = (turns - 1.0) / 31.0;
      keep = keep < 0.0 ? 0.0 : keep > 1.0 ? 1.0 : keep;
      f = keep * f + (1.0 - keep) * f / factor;
    }
    for (int x = 0; x < axes; ++x) freq[x * n + j] = f;
  }
  *amplitude = scaling == RESLIM_ROTARY_BY_PARTS ? static_cast<float>(0.1 * std::log(factor) + 1.0) : 1.0f;
  return RESLIM_OK;
}
