// How a 32-key tile of K and V meets the matrix cores: which key each score register stands for, and the operands of the
// PV product (attention.hip, attend.hip).
#pragma once
#include "common.hpp"

namespace dinfer {

// B operand of the PV product for k-step s2: the G probabilities this lane holds for that step's keys, and
// the matching A operand (V^T of those keys for feature row d).  key_of_row: which of a tile's 32 keys row r of the
// score tile stands for (any assignment will do, as the softmax does not care); key_of_acc: the tile-local key of
// accumulator register v.
template <typename E> struct PvStep;
template <> struct PvStep<bf16_t> {
  // Bits 2 and 3 of the row are swapped, so that the eight registers 8*s2 .. 8*s2+7 of half h hold the consecutive keys
  // 16*s2 + 8h .. +7 and their V^T entries are one 16-byte load (with rows in key order they are two 8-byte loads
  // eight keys apart, twice as many instructions for the address unit).
  static constexpr int STEPS = 2;
  __device__ static int key_of_row(int r) { return (r & 19) | ((r & 4) << 1) | ((r & 8) >> 1); }
  __device__ static int key_of_acc(int v, int half) { return 16 * (v >> 3) + 8 * half + (v & 7); }
  // plane 0: bf16(p); plane 1: bf16(p - plane 0)
  __device__ static bf16x8 p_vec(const float (&p)[16], int s2, int plane) {
    bf16x8 r;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const bf16_t hi = (bf16_t)p[8 * s2 + i];
      r[i] = plane == 0 ? hi : (bf16_t)(p[8 * s2 + i] - (float)hi);
    }
    return r;
  }
  // vrow: V^T row of feature d inside the page of this step (16 slots contiguous)
  __device__ static bf16x8 v_vec(const bf16_t* vrow, int half, int /*s2*/) { return load16<bf16_t>(vrow + 8 * half); }
  __device__ static int page_of_step(int s2) { return s2; }
  __device__ static int key_of(int s2, int half, int i) { return 16 * s2 + 8 * half + i; }
};
template <> struct PvStep<float> {
  // step s2 in {0..3}: registers 4*s2 .. 4*s2+3 -> keys 8*s2 + 4h + {0..3}
  static constexpr int STEPS = 4;
  __device__ static int key_of_row(int r) { return r; }
  __device__ static int key_of_acc(int v, int half) { return acc_row(v, half); }
  __device__ static f32x4 p_vec(const float (&p)[16], int s2, int /*plane*/) {
    f32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = p[4 * s2 + i];
    return r;
  }
  __device__ static f32x4 v_vec(const float* vrow, int half, int s2) {
    return *reinterpret_cast<const f32x4*>(vrow + 8 * (s2 & 1) + 4 * half);
  }
  __device__ static int page_of_step(int s2) { return s2 >> 1; }
  __device__ static int key_of(int s2, int half, int i) { return 8 * s2 + 4 * half + i; }
};

}  // namespace dinfer
