// Host side of the tensor-core products of the operators of heads.
#include "head_mma.cuh"

#include <mutex>
#include <set>
#include <utility>

namespace lc {
namespace ops {

__device__ unsigned long long g_errors;

uint64_t operator_errors(cudaStream_t s) {
  unsigned long long n = 0;
  LC_CUDA(cudaMemcpyFromSymbolAsync(&n, g_errors, sizeof n, 0, cudaMemcpyDeviceToHost, s));
  LC_CUDA(cudaStreamSynchronize(s));
  return n;
}

void allow_smem(const void* kernel, int bytes) {
  static std::mutex mu;
  static std::set<std::pair<int, const void*>> done;
  int dev = 0;
  LC_CUDA(cudaGetDevice(&dev));
  std::lock_guard<std::mutex> lock(mu);
  if (!done.insert({dev, kernel}).second) return;
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e != cudaSuccess) done.erase({dev, kernel});
  LC_CUDA(e);
}

namespace mma {

EncodeTiledFn encoder() {
  static const EncodeTiledFn fn = [] {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult q;
    const cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &q);
    return e == cudaSuccess && q == cudaDriverEntryPointSuccess ? reinterpret_cast<EncodeTiledFn>(f) : nullptr;
  }();
  LC_REQUIRE(fn != nullptr, LIPCACHE_E_CUDA, "cuTensorMapEncodeTiled is unavailable from the driver");
  return fn;
}

int num_sms() {
  static int known[64] = {};
  int dev = 0;
  LC_CUDA(cudaGetDevice(&dev));
  if (dev < 64 && known[dev]) return known[dev];
  int n = 0;
  LC_CUDA(cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev));
  if (dev < 64) known[dev] = n;
  return n;
}

unsigned long long* error_counter() {
  static unsigned long long* known[64] = {};
  int dev = 0;
  LC_CUDA(cudaGetDevice(&dev));
  if (dev < 64 && known[dev]) return known[dev];
  void* p = nullptr;
  LC_CUDA(cudaGetSymbolAddress(&p, g_errors));
  if (dev < 64) known[dev] = static_cast<unsigned long long*>(p);
  return static_cast<unsigned long long*>(p);
}

CUtensorMap tensor_map(const Tensor& t, int box_rows, int box_cols) {
  CUtensorMap map;
  const cuuint64_t dims[3] = {(cuuint64_t)t.cols, (cuuint64_t)t.rows, (cuuint64_t)t.planes};
  const cuuint64_t strides[2] = {(cuuint64_t)t.ld * 2, (cuuint64_t)(t.planes > 1 ? t.plane : t.ld * t.rows) * 2};
  const cuuint32_t box[3] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows, 1}, step[3] = {1, 1, 1};
  // (16-bit elements of either kind: the copy only moves them)
  const CUresult r = encoder()(&map, CU_TENSOR_MAP_DATA_TYPE_UINT16, 3, const_cast<void*>(t.base), dims, strides, box,
                               step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                               box_cols == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
                               CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  LC_REQUIRE(r == CUDA_SUCCESS, LIPCACHE_E_CUDA, "cuTensorMapEncodeTiled failed: " + std::to_string((int)r));
  return map;
}

}  // namespace mma
}  // namespace ops
}  // namespace lc
