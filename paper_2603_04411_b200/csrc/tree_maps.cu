// Row maps of a serving step, made on the GPU from request lengths: slots of new tokens, positions and ancestor masks of drafted
// trees, and the path of a tree that verification keeps.  All three are bound by launch and by one chain of dependent reads; the
// requests' tables are small, so every CTA that needs the requests' offsets scans all lengths itself instead of waiting for another.
// In a graph of 50 calls: slots of 64 requests 2.5 us, of 256 with 131000 rows 4.0, trees of 8 nodes 1.6, 64 trees of 64 nodes 1.8; their paths 2.9 and 4.9.
#include "twkv_dev.h"
#include "tree.h"

namespace twkv {

// Exclusive scan of one 64-bit value per thread over a CTA of 1024 threads (lengths are the caller's: their sum may pass 32 bits).
__device__ __forceinline__ long long block_scan_excl64(long long x, long long* s_warp, long long* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  long long incl = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long u = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += u;
  }
  __syncthreads();                                         // s_warp may still be read from the previous call
  if (lane == 31) s_warp[warp] = incl;
  __syncthreads();
  if (warp == 0) {
    long long w = s_warp[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long u = __shfl_up_sync(0xffffffffu, w, o);
      if (lane >= o) w += u;
    }
    s_warp[lane] = w;
  }
  __syncthreads();
  *total = s_warp[31];
  return (warp ? s_warp[warp - 1] : 0) + incl - x;
}

// offsets[i + 1] = sum of the first i + 1 lengths; row j of request i: its sequence, start + (j - offsets[i]).  Every CTA scans the
// lengths into shared memory, then takes its share of the rows and finds a row's request by bisection.  A call with anything
// invalid writes zero offsets and no row.
__global__ void __launch_bounds__(1024) slot_map_kernel(DevView v, int layer, const int* req_seqs, const int* req_lens, const int* starts, int n_req,
                                                        int max_rows, int* offsets, int* seq_ids, int* positions) {
  extern __shared__ int s_off[];                           // [n_req + 1], then a bit per sequence (no starts given)
  unsigned* s_seen = reinterpret_cast<unsigned*>(s_off + n_req + 1);
  __shared__ long long s_warp[32];
  chain_start();
  chain_wait();
  const int tid = threadIdx.x;
  for (int i = tid; i < (v.S + 31) / 32; i += 1024) s_seen[i] = 0u;
  __syncthreads();
  long long sum = 0;
  int bad = 0;
  for (int i0 = 0; i0 < n_req; i0 += 1024) {
    const int i = i0 + tid;
    long long len = 0;
    if (i < n_req) {
      const int seq = req_seqs[i];
      len = req_lens[i];
      const bool seq_ok = seq >= 0 && seq < v.S;
      long long start = 0;
      if (seq_ok && starts) start = starts[i];
      if (seq_ok && !starts) {
        start = v.stok(layer)[seq];
        if (atomicOr(&s_seen[seq >> 5], 1u << (seq & 31)) >> (seq & 31) & 1u) bad = 1;     // its rows would share positions
      }
      if (!seq_ok || len < 0 || start < 0 || start + len > (long long)ROPE_LO * ROPE_HI) { bad = 1; len = 0; }
    }
    long long total;
    const long long off = sum + block_scan_excl64(len, s_warp, &total);
    sum += total;
    if (i < n_req) s_off[i] = (int)(off < 0x7fffffffll ? off : 0x7fffffffll);
  }
  bad = __syncthreads_or(bad);
  const bool full = sum > max_rows;
  const int n = bad || full ? 0 : (int)sum;
  if (tid == 0) s_off[n_req] = n;
  if (blockIdx.x == 0) {
    for (int i = tid; i <= n_req; i += 1024) offsets[i] = i == n_req ? n : (n ? s_off[i] : 0);
    if (tid == 0 && (bad || full)) set_status(v, bad ? TWKV_ERR_INVALID_ARG : TWKV_ERR_CAPACITY);
  }
  __syncthreads();
  for (int r = blockIdx.x * 1024 + tid; r < n; r += gridDim.x * 1024) {
    int lo = 0, hi = n_req - 1;                            // the last request that starts at or before row r
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (s_off[mid] <= r) lo = mid; else hi = mid - 1;
    }
    const int seq = req_seqs[lo];
    seq_ids[r] = seq;
    positions[r] = (starts ? starts[lo] : v.stok(layer)[seq]) + r - s_off[lo];
  }
}

// A warp per tree, two nodes per lane: masks by pointer doubling, M[j] |= M[up[j]], up[j] = up[up[j]], six rounds for 64 nodes.
__global__ void __launch_bounds__(256) tree_map_kernel(DevView v, const int* offsets, const int* parents, int n_req, int n_rows, int max_nodes,
                                                       int* positions, unsigned long long* masks) {
  __shared__ unsigned long long s_mask[8][TWKV_TREE_MAX_NODES];
  __shared__ int s_up[8][TWKV_TREE_MAX_NODES];
  chain_start();
  chain_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, i = blockIdx.x * 8 + warp;
  if (i >= n_req) return;
  int first, n;
  if (!tree_rows(offsets, i, n_rows, max_nodes, &first, &n)) {
    if (lane == 0) set_status(v, TWKV_ERR_INVALID_ARG);
    return;
  }
  if (n == 0) return;
  const int pos0 = positions[first];
  bool ok = true;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int j = lane + 32 * k;
    const int up = j < n ? parents[first + j] : -1;
    ok = ok && up >= -1 && up < j;
    s_up[warp][j] = up;
    s_mask[warp][j] = 1ull << j;
  }
  if (!__all_sync(0xffffffffu, ok)) {                      // a parent that is not an earlier node of the tree: no node sees anything
    for (int j = lane; j < n; j += 32) masks[first + j] = 0ull;
    if (lane == 0) set_status(v, TWKV_ERR_INVALID_ARG);
    return;
  }
#pragma unroll 1
  for (int round = 0; round < 6; ++round) {
    __syncwarp();
    unsigned long long m[2];
    int up[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int j = lane + 32 * k, u = s_up[warp][j];
      m[k] = u >= 0 ? s_mask[warp][u] : 0ull;
      up[k] = u >= 0 ? s_up[warp][u] : -1;
    }
    __syncwarp();
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      s_mask[warp][lane + 32 * k] |= m[k];
      s_up[warp][lane + 32 * k] = up[k];
    }
  }
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int j = lane + 32 * k;
    if (j >= n) continue;
    const unsigned long long m = s_mask[warp][j];
    masks[first + j] = m;
    if (j > 0) positions[first + j] = pos0 + __popcll(m) - 1;      // (row 0 is the root: it keeps its position)
  }
}

// A warp per tree, two nodes per lane.  The walk goes from a node to its lowest child that carries the node's chosen token; children
// have larger numbers than their parents, so the path in order is the set bits of a word.  The CTA that finishes last lays the paths
// of all requests one behind the other.
__global__ void __launch_bounds__(1024) tree_accept_kernel(DevView v, const int* offsets, const int* parents, const int* draft, const int* target,
                                                           int n_req, int n_rows, int max_nodes, int* n_accepted, int* rows, int* next_tokens,
                                                           unsigned long long* paths, int* ticket) {
  __shared__ long long s_warp[32];
  __shared__ int s_last;
  chain_start();
  chain_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, i = blockIdx.x * 32 + warp;
  if (i < n_req) {
    int first = 0, n = 0;
    if (!tree_rows(offsets, i, n_rows, max_nodes, &first, &n)) {
      if (lane == 0) set_status(v, TWKV_ERR_INVALID_ARG);
      n = 0;
    }
    int up[2], tok[2], want[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int j = lane + 32 * k;
      const bool in = j < n;
      up[k] = in ? parents[first + j] : -1;
      tok[k] = in ? draft[first + j] : 0;
      want[k] = in ? target[first + j] : -1;
    }
    unsigned long long path = 0ull;
    int next = -1;
    for (int cur = n > 0 ? 0 : TWKV_TREE_MAX_NODES; cur < TWKV_TREE_MAX_NODES;) {      // (a child's number is larger: ends after 64 steps)
      path |= 1ull << cur;
      const int w = __shfl_sync(0xffffffffu, cur < 32 ? want[0] : want[1], cur & 31);
      next = w;
      const unsigned lo = __ballot_sync(0xffffffffu, lane < n && lane > cur && up[0] == cur && tok[0] == w);
      const unsigned hi = __ballot_sync(0xffffffffu, lane + 32 < n && lane + 32 > cur && up[1] == cur && tok[1] == w);
      cur = lo ? __ffs(lo) - 1 : hi ? __ffs(hi) + 31 : TWKV_TREE_MAX_NODES;
    }
    if (lane == 0) {
      n_accepted[i] = __popcll(path);
      next_tokens[i] = next;
      paths[i] = path;
    }
  }
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) s_last = gridDim.x == 1 || atomicAdd(ticket, 1) == (int)gridDim.x - 1;
  __syncthreads();
  if (!s_last) return;
  __threadfence();
  if (threadIdx.x == 0 && gridDim.x > 1) *ticket = 0;
  long long sum = 0;
  for (int i0 = 0; i0 < n_req; i0 += 1024) {
    const int j = i0 + threadIdx.x;
    unsigned long long p = j < n_req ? *(volatile unsigned long long*)&paths[j] : 0ull;
    long long total;
    long long at = sum + block_scan_excl64(__popcll(p), s_warp, &total);
    sum += total;
    const int first = p ? offsets[j] : 0;
    for (; p; p &= p - 1ull, ++at)
      if (at < n_rows) rows[at] = first + __ffsll((long long)p) - 1;      // (offsets that overlap could name more rows than there are)
  }
}

cudaError_t launch_slot_map(const DevView& v, int layer, const int* req_seqs, const int* req_lens, const int* starts, int n_req, int max_rows,
                            int* offsets, int* seq_ids, int* positions, int sm_count, cudaStream_t st) {
  ProfScope ps(TWKV_K_PLAN, st);
  const int ctas = (int)(((long long)max_rows + 1023) / 1024);
  const size_t smem = (size_t)(n_req + 1 + (v.S + 31) / 32) * sizeof(int);
  const cudaError_t e = launch_chained(slot_map_kernel, dim3(ctas < 1 ? 1 : ctas > sm_count ? sm_count : ctas), dim3(1024), dim3(1), smem, st, v, layer,
                                       req_seqs, req_lens, starts, n_req, max_rows, offsets, seq_ids, positions);
  if (e != cudaSuccess) return e;
  count_launch();
  return cudaGetLastError();
}

cudaError_t launch_tree_map(const DevView& v, const int* offsets, const int* parents, int n_req, int n_rows, int max_nodes, int* positions,
                            unsigned long long* masks, cudaStream_t st) {
  ProfScope ps(TWKV_K_PLAN, st);
  const cudaError_t e = launch_chained(tree_map_kernel, dim3((n_req + 7) / 8), dim3(256), dim3(1), 0, st, v, offsets, parents, n_req, n_rows, max_nodes,
                                       positions, masks);
  if (e != cudaSuccess) return e;
  count_launch();
  return cudaGetLastError();
}

cudaError_t launch_tree_accept(const DevView& v, const int* offsets, const int* parents, const int* draft, const int* target, int n_req, int n_rows,
                               int max_nodes, int* n_accepted, int* rows, int* next_tokens, cudaStream_t st) {
  ProfScope ps(TWKV_K_PLAN, st);
  // the paths wait in the scratch of a prefill call's tables, the ticket in a word of the status region that is zero between calls
  const cudaError_t e = launch_chained(tree_accept_kernel, dim3((n_req + 31) / 32), dim3(1024), dim3(1), 0, st, v, offsets, parents, draft, target, n_req,
                                       n_rows, max_nodes, n_accepted, rows, next_tokens, reinterpret_cast<unsigned long long*>(v.wave_buf), v.status + 4);
  if (e != cudaSuccess) return e;
  count_launch();
  return cudaGetLastError();
}

}  // namespace twkv
