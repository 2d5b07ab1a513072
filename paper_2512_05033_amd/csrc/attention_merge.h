// Merge of split partials, shared by the attention kernels.
#pragma once

#include "common.h"

#include <math.h>

// Of one (token, head) row: sum_s w_s l_s o_s and sum_s w_s l_s with w_s = exp2(m_s - m), m = max_s m_s and o_s the split's
// normalised result.  Beside a result in fp16 stand m_s + log2(l_s), which is all that the weight needs, and the power of two that it is
// relative to.  A thread owns eight consecutive elements (`piece`) of the row; idx = token * Hq + head, stride = T * Hq.
struct SplitSum {
  float m, l, acc[8];
  __device__ __forceinline__ void clear() {
    m = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = 0.f;
  }
  // Splits first, first + step, ... below n_splits, eight at a time: all their loads go out together (a loop over a run-time count
  // waits for each before it asks for the next), then they are combined under their common maximum; groups of eight are
  // chained by the usual online rescaling.
  // Part: bf16, _Float16 or float.
  template <int HD, typename Part>
  __device__ __forceinline__ void add(const Part *__restrict__ part_acc, const float *__restrict__ part_ml, size_t stride,
                                      size_t idx, int piece, int first, int step, int n_splits) {
    typedef Part part8 __attribute__((ext_vector_type(8)));
    constexpr bool RELATIVE = __is_same(Part, _Float16);
    for (int s0 = first; s0 < n_splits; s0 += 8 * step) {
      float2 ml[8];
      part8 v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int s = s0 + j * step;
        if (s < n_splits) {
          ml[j] = *(const float2 *)(part_ml + (s * stride + idx) * 2);
          v[j] = *(const part8 *)(part_acc + (s * stride + idx) * HD + piece * 8);
        } else {
          ml[j] = float2{-INFINITY, 0.f};
#pragma unroll
          for (int e = 0; e < 8; ++e) v[j][e] = (Part)0.f;
        }
      }
      float m_new = m;
#pragma unroll
      for (int j = 0; j < 8; ++j) m_new = fmaxf(m_new, ml[j].x);
      // No key of any split so far visible to the row, or NaN all of them: the weights are 0 and keep a NaN.
      const float ref = m_new == -INFINITY ? 0.f : m_new, keep = exp2f(m - ref);   // m = -inf: 0
      m = m_new;
      l *= keep;
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] *= keep;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float x = exp2f(ml[j].x - ref), w = RELATIVE ? x : x * ml[j].y, f = x * ml[j].y;   // a split without visible keys: exp2(-inf) * 0 = 0
        l += w;
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] += f * (float)v[j][e];
      }
    }
  }
  // Another thread's sum: m, l and the eight accumulators in a row.
  __device__ __forceinline__ void join(const float *x) {
    const float m_new = fmaxf(m, x[0]);
    const float keep = m == -INFINITY ? 0.f : exp2f(m - m_new), w = x[0] == -INFINITY ? 0.f : exp2f(x[0] - m_new);
    m = m_new;
    l = l * keep + x[1] * w;
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = acc[e] * keep + x[2 + e] * w;
  }
  __device__ __forceinline__ void store(bf16 *dst) const {
    const float inv = 1.0f / l;
    bf16x8 r;
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = (bf16)(acc[e] * inv);
    *(bf16x8 *)dst = r;
  }
};
