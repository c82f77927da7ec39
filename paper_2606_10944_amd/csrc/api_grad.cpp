// C ABI of the gradient of coreset attention: argument validation and launches.
#include <stdint.h>

#include "../../include/thin.h"
#include "grad.hpp"
#include "observe.hpp"

using thin::observed;

namespace {

constexpr int64_t kMaxSlices = 65535;
// Query rows and coreset rows of a call: a row's wave is a launch's thread times 64, which the
// runtime counts in 32 bits.
constexpr int64_t kMaxQueries = (int64_t)1 << 29;
constexpr int64_t kMaxKeys = (int64_t)1 << 25;
// Places of a slice's list: the join compares every one with every other (0.1 s at a million).
constexpr int64_t kMaxList = (int64_t)1 << 18;
constexpr int64_t kMaxRows = (int64_t)1 << 30;

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
bool rows(const void* p) { return p && aligned(p, 16); }

bool known_dtype(int32_t t) { return t == THIN_FP32 || t == THIN_BF16; }

bool valid_sizes(int64_t B, int64_t H, int64_t n_q, int64_t n, int64_t d, int64_t n_out) {
  if (B < 1 || H < 1 || B > kMaxSlices || H > kMaxSlices || B * H > kMaxSlices) return false;
  if (d != 32 && d != 64 && d != 128) return false;
  if (n < 1 || n > kMaxRows || n_q < 1 || n_q > kMaxQueries || n_out < 1 || n_out > kMaxList)
    return false;
  return B * H * n_q <= kMaxQueries && B * H * n_out <= kMaxKeys;
}

}  // namespace

extern "C" {

int thin_attention_backward_plan(int32_t dtype, int64_t B, int64_t H, int64_t n_q, int64_t n,
                                 int64_t d, int64_t n_out, size_t* workspace_bytes) {
  if (!workspace_bytes) return THIN_EINVAL;
  if (!known_dtype(dtype)) return THIN_EDTYPE;
  if (!valid_sizes(B, H, n_q, n, d, n_out)) return THIN_EINVAL;
  *workspace_bytes = 0;
  for (const bool exact : {false, true}) {  // the larger of what either type of dO takes
    const thin::GradShape s = thin::grad_shape(B * H, n_q, n_out, d, dtype == THIN_BF16,
                                               exact && dtype == THIN_BF16);
    const size_t n = thin::grad_bytes(s, B * H, n_q, d, true).all();
    if (n > *workspace_bytes) *workspace_bytes = n;
  }
  return THIN_OK;
}

int thin_attention_backward(const void* Q, const void* K, const void* V, int32_t dtype, int64_t B,
                            int64_t H, int64_t n_q, int64_t n, int64_t d, const int32_t* idx,
                            const float* logw, int64_t n_out, const void* dO, int32_t out_dtype,
                            void* dQ, void* dK, void* dV, float* dlogw, void* workspace,
                            size_t workspace_bytes, void* stream) {
  if (!known_dtype(dtype) || !known_dtype(out_dtype)) return THIN_EDTYPE;
  if (!valid_sizes(B, H, n_q, n, d, n_out)) return THIN_EINVAL;
  if (!rows(Q) || !rows(K) || !rows(V) || !rows(dO) || !rows(dQ) || !rows(dK) || !rows(dV) ||
      !idx || !aligned(idx, 4) || !aligned(logw, 4) || !aligned(dlogw, 4))
    return THIN_EINVAL;
  const void* outs[] = {dQ, dK, dV, dlogw};
  const void* ins[] = {Q, K, V, dO, idx, logw};
  for (int i = 0; i < 4; ++i) {
    for (const void* in : ins)
      if (outs[i] && outs[i] == in) return THIN_EINVAL;
    for (int j = 0; j < i; ++j)
      if (outs[i] && outs[i] == outs[j]) return THIN_EINVAL;
  }
  thin::GradArgs a{};
  a.shape = thin::grad_shape(B * H, n_q, n_out, d, dtype == THIN_BF16,
                             dtype == THIN_BF16 && out_dtype == THIN_FP32 && dlogw);
  const thin::GradBytes bytes = thin::grad_bytes(a.shape, B * H, n_q, d, true);
  if (!workspace || workspace_bytes < bytes.all() || !aligned(workspace, 256))
    return THIN_EWORKSPACE;
  a.Q = Q;
  a.K = K;
  a.V = V;
  a.dO = dO;
  a.idx = idx;
  a.logw = logw;
  a.dQ = dQ;
  a.dK = dK;
  a.dV = dV;
  a.dlogw = dlogw;
  a.S = B * H;
  a.n = n;
  a.n_q = n_q;
  a.n_out = n_out;
  const int64_t row_bytes = d * (dtype == THIN_BF16 ? 2 : 4);
  a.zeros = thin::grad_zeros(a.shape, n_q, n, row_bytes);
  char* w = static_cast<char*>(workspace);
  a.part = reinterpret_cast<float*>(w);
  if (dlogw) a.part_w = reinterpret_cast<float*>(w + bytes.part);
  a.stats = reinterpret_cast<float*>(w + bytes.part + bytes.part_w);
  hipStream_t st = static_cast<hipStream_t>(stream);
  hipError_t e = hipSuccess;
  if (a.zeros)
    e = observed(THIN_KERNEL_ATTENTION_GRAD, -1, st,
                 [&] { return thin::launch_grad_zeros(row_bytes, a, st); });
  if (e == hipSuccess && !a.shape.one)
    e = observed(THIN_KERNEL_ATTENTION_GRAD, -1, st,
                 [&] { return thin::launch_grad_rows(dtype, out_dtype, d, a, st); });
  if (e == hipSuccess)
    e = observed(THIN_KERNEL_ATTENTION_GRAD, -1, st,
                 [&] { return thin::launch_grad_keys(dtype, out_dtype, d, a, st); });
  if (e == hipSuccess)
    e = observed(THIN_KERNEL_ATTENTION_GRAD, -1, st,
                 [&] { return thin::launch_grad_join(dtype, d, a, st); });
  return e == hipSuccess ? THIN_OK : THIN_EHIP;
}

}  // extern "C"
