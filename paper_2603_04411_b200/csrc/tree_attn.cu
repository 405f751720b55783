// Attention of drafted trees over the mixed-rank cache: scores, weighted values, projection.
//
//   tree_plan_kernel (tree_plan.cu)  lists, splits, links, the nodes' states and the queries as operands
//   tree_score_kernel (tree_score.cu)  per K tile and KV head: keys rebuilt and rotated (Eq. 3), scores with all query rows of the request
//   tree_value_kernel   per (request, split): sum of exp(s - max) X^_V in spectral space, and the sum of the weights
//   tree_merge_kernel   sum of the splits, projection by U_V^-1
#include "twkv_dev.h"
#include "mma_util.cuh"
#include "tree.h"

namespace twkv {

// CTA = (request, split; 64 score columns; panel of 64 components).
template <bool BF16>
__global__ void __launch_bounds__(256) tree_value_kernel(DevView v, TreeCall a) {
  __shared__ float s_p[TILE][64];
  __shared__ unsigned short s_x[TILE][64];
  chain_start();
  chain_wait();
  const int i = blockIdx.x / a.n_splits, split = blockIdx.x % a.n_splits, c0 = blockIdx.y * 64, panel = blockIdx.z, tid = threadIdx.x;
  const int* cut = a.vcut + (size_t)i * (a.n_splits + 1) + split;
  const int col = tid & 63, j0 = (tid >> 6) * 16;
  float m = c0 + col < a.C ? dec_ordered(a.seqmax[(size_t)i * a.C + c0 + col]) : 0.f;
  if (m == -INFINITY) m = 0.f;
  float acc[16], l = 0.f;
  for (int k = 0; k < 16; ++k) acc[k] = 0.f;
  for (int k = cut[0]; k < cut[1]; ++k) {
    const int4 d = a.vmeta[(size_t)i * (v.TPS + 1) + k];
    if (panel > 0 && d.y <= panel) continue;
    __syncthreads();
    for (int t = tid >> 6; t < TILE; t += 4) {
      s_p[t][col] = t < d.z && c0 + col < a.C ? expf(a.scores[((size_t)d.x * TILE + t) * a.C + c0 + col] - m) : 0.f;
      const unsigned char* src = d.w < 0 ? a.nv + ((size_t)i * v.NC + panel) * TREE_PANEL_ROWS * PANEL * 2 : v.blocks + (size_t)(d.w + panel) * BLOCK_BYTES;
      s_x[t][col] = t < d.z ? reinterpret_cast<const unsigned short*>(src)[t * PANEL + col] : 0;
    }
    __syncthreads();
    for (int t = 0; t < d.z; ++t) {
      const float p = s_p[t][col];
      l += p;
      for (int e = 0; e < 16; ++e) acc[e] += p * to_f32<BF16>(s_x[t][j0 + e]);
    }
  }
  const int c = c0 + col, g = c / a.Rs, n = c % a.Rs;
  if (c >= a.C || n >= a.R) return;
  const size_t part = (((size_t)i * a.T + n / v.rep) * a.n_splits + split) * v.Hq + g * v.rep + n % v.rep;
  for (int e = 0; e < 16; ++e) a.part_acc[part * v.d_kv + panel * PANEL + j0 + e] = acc[e];
  if (panel == 0 && j0 == 0) a.part_l[part] = l;
}

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

cudaError_t launch_tree_value(const DevView& v, const TreeCall& a, cudaStream_t st) {
  ProfScope ps(TWKV_K_VACC, st);
  auto kernel = v.dtype == TWKV_BF16 ? tree_value_kernel<true> : tree_value_kernel<false>;
  const cudaError_t e = launch_chained(kernel, dim3(a.n_req * a.n_splits, (a.C + 63) / 64, v.NC), dim3(256), dim3(1), 0, st, v, a);
  if (e != cudaSuccess) return e;
  count_launch();
  return cudaGetLastError();
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
