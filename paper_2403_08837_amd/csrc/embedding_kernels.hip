// Embedding: rows of a table by token ids, scaled, and the gradient of the table.
#include "elem.h"
#include "kernels.h"

namespace cdp {

namespace {

template <typename T>
__global__ __launch_bounds__(256) void embedding_fwd_kernel(const T* table, const int32_t* ids, T* out, float scale, int vocab, int C) {
  const int64_t t = blockIdx.x;
  const int id = ids[t];
  const bool in = id >= 0 && id < vocab;
  for (int c = threadIdx.x; c < C; c += 256) st_f32<T>(out, t * C + c, in ? scale * ld_f32<T>(table, (int64_t)id * C + c) : 0.f);
}

// One workgroup per row of the table: its tokens in ascending order.
template <typename T>
__global__ __launch_bounds__(256) void embedding_bwd_kernel(const int32_t* ids, const T* dout, float* dtable, float scale, int accumulate, int rows, int C) {
  const int64_t v = blockIdx.x;
  for (int c0 = 0; c0 < C; c0 += 256) {
    const int c = c0 + threadIdx.x;
    float sum = 0.f;
    bool any = false;
    for (int t = 0; t < rows; ++t) {
      if (ids[t] != (int)v) continue;
      any = true;
      if (c < C) sum += ld_f32<T>(dout, (int64_t)t * C + c);
    }
    if (c < C && (any || !accumulate)) dtable[v * C + c] = scale * sum + (accumulate ? dtable[v * C + c] : 0.f);
  }
}

}  // namespace

hipError_t launch_embedding_fwd(const void* table, const int32_t* ids, void* out, float scale, int rows, int vocab, int C, int dtype,
                                hipStream_t stream) {
  if (dtype == DT_BF16)
    hipLaunchKernelGGL((embedding_fwd_kernel<uint16_t>), dim3(rows), dim3(256), 0, stream, static_cast<const uint16_t*>(table), ids,
                       static_cast<uint16_t*>(out), scale, vocab, C);
  else
    hipLaunchKernelGGL((embedding_fwd_kernel<float>), dim3(rows), dim3(256), 0, stream, static_cast<const float*>(table), ids,
                       static_cast<float*>(out), scale, vocab, C);
  return hipGetLastError();
}

int64_t embedding_bwd_workspace_bytes(int rows, int C) { return 16ll * rows + 8ll * C * ((rows + 31ll) / 32) + 512; }

hipError_t launch_embedding_bwd(const int32_t* ids, const void* dout, float* dtable, float scale, void*, bool accumulate, int rows, int vocab, int C,
                                int dtype, hipStream_t stream) {
  if (dtype == DT_BF16)
    hipLaunchKernelGGL((embedding_bwd_kernel<uint16_t>), dim3(vocab), dim3(256), 0, stream, ids, static_cast<const uint16_t*>(dout), dtable, scale,
                       accumulate, rows, C);
  else
    hipLaunchKernelGGL((embedding_bwd_kernel<float>), dim3(vocab), dim3(256), 0, stream, ids, static_cast<const float*>(dout), dtable, scale, accumulate,
                       rows, C);
  return hipGetLastError();
}

}  // namespace cdp
