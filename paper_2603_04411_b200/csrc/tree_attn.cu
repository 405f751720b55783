// Attention of drafted trees over the mixed-rank cache: scores, weighted values, projection.
//
//   tree_plan_kernel (tree_plan.cu)  lists, splits, links, the nodes' states and the queries as operands
//   tree_score_kernel (tree_score.cu)  per K tile and KV head: keys rebuilt and rotated (Eq. 3), scores with all query rows of the request
//   tree_value_kernel (tree_value.cu)  per (request, split): sum of exp(s - max) X^_V in spectral space, and the sum of the weights
//   tree_merge_kernel   sum of the splits, projection by U_V^-1
#include "twkv_dev.h"
#include "mma_util.cuh"
#include "tree.h"

namespace twkv {

// CTA = (request, node; query head).
template <bool BF16>
__global__ void __launch_bounds__(128) tree_merge_kernel(DevView v, TreeCall a, const unsigned short* U) {
  extern __shared__ float s_acc[];                         // [d_kv]
  chain_start();
  chain_wait();
  const int i = blockIdx.x / a.T, t = blockIdx.x % a.T, head = blockIdx.y, tid = threadIdx.x;
  const int4 info = a.info[i];
  if (t >= info.y) return;
  float l = 0.f;
  for (int j = tid; j < v.d_kv; j += 128) s_acc[j] = 0.f;
  if (info.z >= 0) {
    const size_t p0 = ((size_t)blockIdx.x * a.n_splits) * v.Hq + head;
    for (int s = 0; s < a.n_splits; ++s) {
      l += a.part_l[p0 + (size_t)s * v.Hq];
      const int* cut = a.vcut + (size_t)i * (a.n_splits + 1) + s;
      if (cut[1] > cut[0])                                 // (an empty split's part is not written)
        for (int j = tid; j < v.d_kv; j += 128) s_acc[j] += a.part_acc[(p0 + (size_t)s * v.Hq) * v.d_kv + j];
    }
  }
  __syncthreads();
  float o = 0.f;
  for (int j = 0; j < v.d_kv; ++j) o += s_acc[j] * to_f32<BF16>(U[(size_t)j * v.d_kv + (head / v.rep) * HEAD_DIM + tid]);
  o = l == 0.f ? 0.f : o / l;
  if (info.z >= 0 && (a.masks[info.x + t] & a.bad[i])) o = NAN;
  const size_t at = ((size_t)(info.x + t) * v.Hq + head) * HEAD_DIM + tid;
  if (v.out_dtype == TWKV_F32) reinterpret_cast<float*>(a.out)[at] = o;
  else if (v.out_dtype == TWKV_BF16) reinterpret_cast<unsigned short*>(a.out)[at] = from_f32<true>(o);
  else reinterpret_cast<unsigned short*>(a.out)[at] = from_f32<false>(o);
}

cudaError_t launch_tree_merge(const DevView& v, const TreeCall& a, const LayerParams& lp, cudaStream_t st) {
  ProfScope ps(TWKV_K_MERGE, st);
  auto kernel = v.dtype == TWKV_BF16 ? tree_merge_kernel<true> : tree_merge_kernel<false>;
  const cudaError_t e = launch_chained(kernel, dim3(a.n_req * a.T, v.Hq), dim3(128), dim3(1), v.d_kv * sizeof(float), st, v, a,
                                       reinterpret_cast<const unsigned short*>(lp.Uinv_v));
  if (e != cudaSuccess) return e;
  count_launch();
  return cudaGetLastError();
}

}  // namespace twkv
