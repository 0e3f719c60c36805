// Device functions of the microscaled kernels by themselves, for test_gpu_mx_device.py.
#include "../paper_2509_24416_gb300/csrc/mx_device.cuh"

namespace {

// Warps 2 p and 2 p + 1 are a pair.  Each goes through its turns until the pair no longer
// agrees to go on; turns[w]: how many it made.  votes: [n][warps].
__global__ void pair_kernel(const int32_t* votes, int n, int32_t* turns) {
  const int warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  int i = 0;
  for (; i < n; ++i) {
    if (!clq::mx::pair_all(1 + (warp >> 1), votes[i * warps + warp] != 0)) break;
    clq::mx::pair_barrier(1 + (warp >> 1));
  }
  if ((threadIdx.x & 31) == 0) turns[warp] = i;
}

// y: GELU of x, or of pairs (gate, up) SwiGLU, two values a thread as the kernels take them.
__global__ void activation_kernel(const float2* x, const float2* up, int n, float2* y) {
  const int i = blockIdx.x * blockDim.x + threadIdx.x;
  if (i < n) y[i] = up == nullptr ? clq::mx::gelu_fast(x[i]) : clq::mx::swiglu_fast(x[i], up[i]);
}

}  // namespace

extern "C" int run_activation(const float2* x, const float2* up, int n, float2* y) {
  activation_kernel<<<(n + 255) / 256, 256>>>(x, up, n, y);
  return cudaDeviceSynchronize();
}

extern "C" int run_pairs(const int32_t* votes, int n, int warps, int32_t* turns) {
  pair_kernel<<<1, 32 * warps>>>(votes, n, turns);
  return cudaDeviceSynchronize();
}
