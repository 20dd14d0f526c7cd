// Softmax cross entropy and its gradient.
#include "operators.cuh"

namespace lc {
namespace ops {
namespace {

// The running maximum m and sum s of exp(z - m); m = -inf, s = 0 is empty.
__device__ __forceinline__ void join(float& m, float& s, float m2, float s2) {
  const float top = fmaxf(m, m2);
  // (an empty side adds nothing; -inf minus itself would be NaN)
  const float a = m == -INFINITY ? 0.f : s * __expf(m - top);
  const float b = m2 == -INFINITY ? 0.f : s2 * __expf(m2 - top);
  m = top;
  s = a + b;
}

template <typename T>
__global__ void __launch_bounds__(256)
    k_cross_entropy(const T* z, int64_t ldz, int classes, const int32_t* target, const float* weight, float* loss,
                    T* dz, int64_t ldd) {
  __shared__ float sm[8], ss[8];
  __shared__ int snan;
  const int64_t row = blockIdx.x;
  const T* zr = z + row * ldz;
  const int y = target[row];
  const bool live = y >= 0 && y < classes;
  if (!live) {
    if (loss && threadIdx.x == 0) loss[row] = 0.f;
    if (dz)
      for (int j = threadIdx.x; j < classes; j += 256) dz[row * ldd + j] = from_f32<T>(0.f);
    return;
  }
  const float w = weight ? weight[row] : 1.f;
  if (threadIdx.x == 0) snan = 0;
  __syncthreads();
  float m = -INFINITY, s = 0.f;
  bool bad = false;
  for (int j = threadIdx.x; j < classes; j += 256) {
    const float v = to_f32<T>(zr[j]);
    bad |= !(v < INFINITY);
    if (j != y) join(m, s, v, 1.f);
  }
  if (bad) snan = 1;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float m2 = __shfl_xor_sync(0xffffffffu, m, o), s2 = __shfl_xor_sync(0xffffffffu, s, o);
    join(m, s, m2, s2);
  }
  if ((threadIdx.x & 31) == 0) sm[threadIdx.x >> 5] = m, ss[threadIdx.x >> 5] = s;
  __syncthreads();
  m = sm[0], s = ss[0];
  for (int i = 1; i < 8; ++i) join(m, s, sm[i], ss[i]);
  const float nan = snan ? NAN : 0.f;
  // The target joins last: 1 - p_y is the others' share, without cancellation.
  const float zy = to_f32<T>(zr[y]);
  __syncthreads();  // dz may be z: the target's logit is read by then
  const float m_o = m, s_o = s;
  join(m, s, zy, 1.f);
  const float others = s_o == 0.f ? 0.f : s_o * __expf(m_o - m) / s;
  if (loss && threadIdx.x == 0) {
    const float l = zy == -INFINITY ? INFINITY : logf(s) + m - zy;
    loss[row] = (w == 0.f ? 0.f : w * l) + nan;
  }
  if (!dz) return;
  const float inv = m == -INFINITY ? 0.f : 1.f / s;
  for (int j = threadIdx.x; j < classes; j += 256) {
    const float v = to_f32<T>(zr[j]);
    const float g = j == y ? -others : v == -INFINITY ? 0.f : __expf(v - m) * inv;
    dz[row * ldd + j] = from_f32<T>(w * g + nan);
  }
}

template <typename T>
void launch(const void* z, int64_t ldz, int64_t tokens, int classes, const int32_t* target, const float* weight,
            float* loss, void* dz, int64_t ldd, cudaStream_t s) {
  k_cross_entropy<T><<<(unsigned)tokens, 256, 0, s>>>(static_cast<const T*>(z), ldz, classes, target, weight, loss,
                                                      static_cast<T*>(dz), ldd);
  LC_LAUNCH_CHECK("k_cross_entropy");
}

}  // namespace

void cross_entropy(int type, const void* z, int64_t ldz, int64_t tokens, int classes, const int32_t* target,
                   const float* weight, float* loss, void* dz, int64_t ldd, cudaStream_t s) {
  if (type == LIPCACHE_F32)
    launch<float>(z, ldz, tokens, classes, target, weight, loss, dz, ldd, s);
  else
    launch<__nv_bfloat16>(z, ldz, tokens, classes, target, weight, loss, dz, ldd, s);
}

}  // namespace ops
}  // namespace lc
