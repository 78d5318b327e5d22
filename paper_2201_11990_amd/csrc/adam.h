// What the optimizer's calls on one tensor and on many share: the sum of a workgroup, the Adam update of one parameter, its host side.
#pragma once
#include <math.h>

#include "common.h"

namespace mtnlg {

// the sum over the workgroup, in thread 0: a fixed tree
template <int THREADS>
__device__ __forceinline__ double workgroup_sum(double s) {
  __shared__ double red[THREADS / 64];
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) s += __shfl_xor(s, off, 64);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  s = red[0];
#pragma unroll
  for (int w = 1; w < THREADS / 64; ++w) s += red[w];
  return s;
}

struct AdamArgs {
  float lr, beta1, beta2, eps, wd, max_norm;
  float inv_c1, inv_c2;   // 1 / (1 - beta1^t), 1 / (1 - beta2^t)
};

__device__ __forceinline__ void adam_one(const AdamArgs &a, float coef, float g, float &p, float &m, float &v) {
  g *= coef;
  m = a.beta1 * m + (1.0f - a.beta1) * g;
  v = a.beta2 * v + (1.0f - a.beta2) * g * g;
  const float mh = m * a.inv_c1, vh = v * a.inv_c2;
  p = p - a.lr * (mh / (sqrtf(vh) + a.eps) + a.wd * p);
}

inline bool adam_desc_ok(const mtnlg_adam_desc &d) {
  return d.step >= 1 && d.beta1 >= 0.0f && d.beta1 < 1.0f && d.beta2 >= 0.0f && d.beta2 < 1.0f && d.eps > 0.0f;
}
inline AdamArgs adam_args(const mtnlg_adam_desc &d) {
  return AdamArgs{d.lr, d.beta1, d.beta2, d.eps, d.weight_decay, d.max_grad_norm, (float)(1.0 / (1.0 - pow((double)d.beta1, (double)d.step))),
                  (float)(1.0 / (1.0 - pow((double)d.beta2, (double)d.step)))};
}

}  // namespace mtnlg
