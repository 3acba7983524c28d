// The norm over all gradients of a model, and the gradients scaled to at most a given norm.
#include "elem.h"
#include "kernels.h"

#include <algorithm>

namespace cdp {

namespace {

constexpr int CLIP_GROUPS = 1024, CLIP_TENSORS = 128;

struct ClipTable {
  const void* g[CLIP_TENSORS];
  void* out[CLIP_TENSORS];
  int64_t count[CLIP_TENSORS];
  int n;
};

// Sum of squares of a workgroup's elements of all tensors of the table, added to part[workgroup] (the first table's: written).
template <typename T> __global__ __launch_bounds__(256) void grad_norm_kernel(const ClipTable t, double* part, int first) {
  __shared__ double lds[256];
  double s = 0;
  for (int i = 0; i < t.n; ++i)
    for (int64_t e = blockIdx.x * 256ll + threadIdx.x; e < t.count[i]; e += CLIP_GROUPS * 256ll) {
      const double v = ld_f32<T>(static_cast<const T*>(t.g[i]), e);
      s += v * v;
    }
  lds[threadIdx.x] = s;
  __syncthreads();
  for (int n = 128; n > 0; n >>= 1) {
    if ((int)threadIdx.x < n) lds[threadIdx.x] += lds[threadIdx.x + n];
    __syncthreads();
  }
  if (threadIdx.x == 0) part[blockIdx.x] = lds[0] + (first ? 0.0 : part[blockIdx.x]);
}
template <typename T> __global__ __launch_bounds__(256) void grad_scale_kernel(const ClipTable t, const double* part, float* norm, float max_norm, int scale) {
  double s = 0;
  for (int i = 0; i < CLIP_GROUPS; ++i) s += part[i];
  const double r = sqrt(s);
  if (blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)r;
  if (!scale) return;
  const float c = r > max_norm ? (float)(max_norm / r) : 1.f;
  for (int i = 0; i < t.n; ++i)
    for (int64_t e = blockIdx.x * 256ll + threadIdx.x; e < t.count[i]; e += gridDim.x * 256ll)
      st_f32<T>(static_cast<T*>(t.out[i]), e, c * ld_f32<T>(static_cast<const T*>(t.g[i]), e));
}

template <typename T>
hipError_t clip(int tensors, const void* const* grads, void* const* outs, const int64_t* counts, float max_norm, float* norm, double* part, hipStream_t stream) {
  for (int pass = 0; pass < 2; ++pass)
    for (int i0 = 0; i0 < tensors; i0 += CLIP_TENSORS) {
      ClipTable t;
      t.n = std::min(CLIP_TENSORS, tensors - i0);
      for (int i = 0; i < t.n; ++i) {
        t.g[i] = grads[i0 + i];
        t.out[i] = outs ? outs[i0 + i] : nullptr;
        t.count[i] = counts[i0 + i];
      }
      if (!pass) hipLaunchKernelGGL((grad_norm_kernel<T>), dim3(CLIP_GROUPS), dim3(256), 0, stream, t, part, i0 == 0);
      else hipLaunchKernelGGL((grad_scale_kernel<T>), dim3(outs ? 2048 : 1), dim3(256), 0, stream, t, part, norm, max_norm, outs != nullptr);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
  return hipSuccess;
}

}  // namespace

hipError_t launch_grad_clip(int tensors, const void* const* grads, void* const* outs, const int64_t* counts, float max_norm, float* norm,
                            void* workspace, int dtype, hipStream_t stream) {
  double* part = static_cast<double*>(workspace);
  return dtype == DT_BF16 ? clip<uint16_t>(tensors, grads, outs, counts, max_norm, norm, part, stream)
                          : clip<float>(tensors, grads, outs, counts, max_norm, norm, part, stream);
}

}  // namespace cdp
