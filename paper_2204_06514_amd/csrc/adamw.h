// What the AdamW kernels share: streaming stores, the scalars of a step.
#pragma once
#include <math.h>

#include "fax_internal.h"

namespace fax {

// Streaming stores for values this kernel does not read again.
__device__ __forceinline__ void nt_store4(float4* p, float4 v) {
  typedef __attribute__((ext_vector_type(4))) float f4;
  const f4 x = {v.x, v.y, v.z, v.w};
  __builtin_nontemporal_store(x, reinterpret_cast<f4*>(p));
}
__device__ __forceinline__ void nt_store2(uint2* p, uint2 v) {
  typedef __attribute__((ext_vector_type(2))) unsigned u2;
  const u2 x = {v.x, v.y};
  __builtin_nontemporal_store(x, reinterpret_cast<u2*>(p));
}

struct AdamScalars {
  float b1, b2, one_m_b1, one_m_b2, inv_bc1, inv_bc2, lr, eps, decay;
};

inline AdamScalars adam_scalars(const FaxAdamW& hp, int step) {
  AdamScalars a;
  a.b1 = (float)hp.beta1; a.b2 = (float)hp.beta2;
  a.one_m_b1 = (float)(1.0 - hp.beta1); a.one_m_b2 = (float)(1.0 - hp.beta2);
  a.inv_bc1 = (float)(1.0 / (1.0 - pow(hp.beta1, (double)step)));
  a.inv_bc2 = (float)(1.0 / (1.0 - pow(hp.beta2, (double)step)));
  a.lr = (float)hp.lr; a.eps = (float)hp.eps;
  a.decay = (float)(1.0 - hp.lr * hp.wd);
  return a;
}

}  // namespace fax
