// Turning rows by their positions: the plain cache's turn (Turn), and what the kernels that norm rows first share with it (packing,
// the shape of a workgroup).  Those take their sines from LDS, where each is formed once and from two floats; Turn's are a function of one
// float and off by up to 2^-22, so the same row may be rounded the other way there.
#pragma once

#include "wave_common.h"

namespace wave {

// ----------------------------------------------------------------------------
// Rotary positions.  A work item is two 16-byte chunks of a row that hold EPC whole pairs (channels i .. and
// i + rot / 2 .. for halves, two neighbouring chunks for neighbours) or, behind the rotated channels, two chunks
// that are copied.  A thread keeps the sines and cosines of its item of one token and goes through the heads with
// them: they cost about forty instructions a pair (the angle in fp64), the turn itself six.
// ----------------------------------------------------------------------------
template <typename T>
__device__ __forceinline__ uint4 pack(const float (&f)[Elem<T>::EPC]);
template <>
__device__ __forceinline__ uint4 pack<float>(const float (&f)[4]) {
  return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
}
template <>
__device__ __forceinline__ uint4 pack<bf16_t>(const float (&f)[8]) {
  typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
  bf16x8 v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (__bf16)f[i];  // nearest even
  return __builtin_bit_cast(uint4, v);
}

template <typename T, int D>
struct Turn {
  static constexpr int EPC = Elem<T>::EPC;
  static constexpr int ITEMS = D / (2 * EPC);  // work items of a row
  float c[EPC], s[EPC];
  int one, two;  // the item's chunks
  bool turns;

  __device__ __forceinline__ void place(const RotaryArgs& r, int item) {
    const int rotated = r.rot / (2 * EPC);
    turns = item < rotated;
    const bool halves = turns && r.pairing == WAVE_ROTARY_HALVES;
    one = halves ? item : 2 * item;
    two = halves ? item + rotated : 2 * item + 1;
  }
  // position(axis) of the item's token; a circle is `1` in turns, so the nearest whole number of circles comes off
  // without error
  template <typename F>
  __device__ __forceinline__ void angles(const RotaryArgs& r, int item, F&& position) {
#pragma unroll
    for (int e = 0; e < EPC; ++e) {
      c[e] = 1.f;
      s[e] = 0.f;
      if (turns) {
        const int i = item * EPC + e;
        const double t = (double)position(r.axis[i]) * r.turns[i];
        sincospif((float)(2.0 * (t - rint(t))), &s[e], &c[e]);
      }
    }
  }
  // the item's two chunks as numbers
  __device__ __forceinline__ void turn(const RotaryArgs& r, float (&x)[EPC], float (&y)[EPC]) const {
    if (r.pairing == WAVE_ROTARY_HALVES) {
#pragma unroll
      for (int e = 0; e < EPC; ++e) {
        const float u = x[e] * c[e] - y[e] * s[e], v = x[e] * s[e] + y[e] * c[e];
        x[e] = u;
        y[e] = v;
      }
    } else {
#pragma unroll
      for (int e = 0; e < EPC; e += 2) {
        const int p = e / 2, h = EPC / 2 + p;  // pairs of the first and of the second chunk
        const float u = x[e] * c[p] - x[e + 1] * s[p], v = x[e] * s[p] + x[e + 1] * c[p];
        const float w = y[e] * c[h] - y[e + 1] * s[h], z = y[e] * s[h] + y[e + 1] * c[h];
        x[e] = u;
        x[e + 1] = v;
        y[e] = w;
        y[e + 1] = z;
      }
    }
  }
  __device__ __forceinline__ void apply(const RotaryArgs& r, uint4& a, uint4& b) const {
    if (!turns) return;
    float x[EPC], y[EPC];
    unpack<T>(a, x);
    unpack<T>(b, y);
    turn(r, x, y);
    a = pack<T>(x);
    b = pack<T>(y);
  }
};

// The threads of a workgroup: ITEMS a row, then `lanes` heads side by side, then the tokens.  A prompt takes one lane
// (a wave then reads whole neighbouring rows of one head), a decode step as many as there are.
struct TurnShape {
  int lane_shift;   // log2 of the heads side by side
  int tokens;       // tokens of a workgroup
  int head_groups;  // workgroups that share the heads of a tile of tokens
};
template <int ITEMS>
inline TurnShape turn_shape(int n, int B, int heads) {
  TurnShape t{0, 256 / ITEMS, 1};
  while (t.tokens > 1 && t.tokens / 2 >= n) {
    t.tokens /= 2;
    ++t.lane_shift;
  }
  // A workgroup's chain of heads is split while the launch leaves most CUs without work.
  const long long tiles = (long long)B * ((n + t.tokens - 1) / t.tokens);
  while (tiles * t.head_groups < 1024 && (heads >> t.lane_shift) > 4 * t.head_groups) t.head_groups *= 2;
  return t;
}

constexpr int TURN_BATCH = 4;  // heads whose loads are in flight together

}  // namespace wave
