// Weighted values of drafted trees on the 5th-generation tensor cores.
//
// As in a decode pass (vacc_tc.cu) the weighted sum is taken in spectral space:
//   acc[j][c] = sum over the split's tokens t of X^_V[t][j] p[t][c],   p = exp(s - top[c]),   l[c] = sum of p[t][c]
// for 64 columns c = (KV head, node, head of the group) per CTA.  Two panels of a V tile are the A operand (M = 128 spectral columns, as TMA
// lands them: MN-major), the weights of 16 tokens and 64 columns the B operand.  Weights go in as two parts of the cache type, both into one
// accumulator (64 columns of tensor memory per pair of panels: 512 for d_kv = 1024), so that a CTA serves twice the columns of a decode CTA
// and the panels are read from L2 half as often.
// The scores of a tile are read a tile ahead into registers (thread = one column, 32 tokens): 32 lanes read 32 columns of a token, a whole
// line, and no room in shared memory goes to them.
// What a column's weights are relative to, top[c], is the largest score so far, moved only when it would grow by more than 2^8 (f16 holds 2^15):
// the sums in tensor memory are rescaled seldom, by the weight warps themselves.  The merge brings the splits' parts together.
// Tiles that are at most half full, and the nodes' tile, are read by the boxes of sixteen rows that hold tokens.
//
// Warp roles (320 threads, one CTA per SM): 0 TMA producer of V panels, 1 MMA issuer (owns the TMEM allocation), 2-9 weights, then the read-out.
// All waits are bounded (tc_util.cuh); a wait that runs out ends the kernel with TWKV_ERR_TIMEOUT.
#include "twkv_dev.h"
#include "tc_util.cuh"
#include "mma_util.cuh"
#include "tree.h"

namespace twkv {
using namespace tc;

constexpr int TV_PWARPS = 8, TV_PTHREADS = 32 * TV_PWARPS, TV_THREADS = 64 + TV_PTHREADS;
constexpr int TV_N = 64;                                       // score columns of a CTA
constexpr int TV_META = 256;                                   // tiles whose descriptors are staged in shared memory at a time
constexpr int TV_STAGES = 4;
constexpr uint32_t TV_PANEL = 16384, TV_STAGE = 2 * TV_PANEL;
constexpr uint32_t TV_ZERO = 2048;                             // 16 token rows of zeros: the missing partner of a lone panel
constexpr uint32_t TV_P_PART = TV_N * 128, TV_P_HALF = 2 * TV_P_PART, TV_P_BUF = 2 * TV_P_HALF;      // [2 halves of 64 tokens][high, low][64 columns][64 tokens]
constexpr uint32_t TV_SMEM = TV_STAGES * TV_STAGE + TV_ZERO + 2 * TV_P_BUF + TV_META * 16 + 2 * TV_PTHREADS * 4 + TV_N * 4 + 256 + 1024;
static_assert(TV_SMEM > CHAIN_TMEM_SMEM && TV_SMEM <= 232448, "no other CTA with tensor memory beside this one");
constexpr int TV_OUT = 32;                                     // columns of the partial result on their way out at a time
static_assert(TV_OUT * TWKV_MAX_CLASSES * PANEL * 4 <= (int)(TV_STAGES * TV_STAGE), "the partial sums leave through the ring's memory");

constexpr float TV_LOG2E = 1.44269504088896340736f;
__device__ __forceinline__ uint64_t tv_pack(float a, float b) { uint64_t r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ void tv_unpack(uint64_t v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t tv_fma2(uint64_t a, uint64_t b, uint64_t c) { uint64_t r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }
__device__ __forceinline__ uint64_t tv_add2(uint64_t a, uint64_t b) { uint64_t r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ float tv_ex2(float x) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }

template <bool BF16>
__global__ void __launch_bounds__(TV_THREADS, 1)
tree_value_kernel(const __grid_constant__ CUtensorMap map_blocks, const __grid_constant__ CUtensorMap map_boxes, const __grid_constant__ CUtensorMap map_nodes,
                  DevView v, TreeCall a) {
  chain_start();
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int d_kv = v.d_kv;
  const int req = blockIdx.x / a.n_splits, split = blockIdx.x - req * a.n_splits, c0 = blockIdx.y * TV_N;
  // shared memory: ring | zero block | weights [2 buffers] | descriptors | row sums | maxima, factors | barriers
  const uint32_t s0 = smem_addr(smem_raw);
  const uint32_t pad = (1024u - (s0 & 1023u)) & 1023u;          // operand tiles need 1024-byte alignment for the swizzle
  unsigned char* base_ptr = smem_raw + pad;
  const uint32_t sRing = s0 + pad, sZero = sRing + TV_STAGES * TV_STAGE, sP = sZero + TV_ZERO;
  unsigned char* sP_ptr = base_ptr + TV_STAGES * TV_STAGE + TV_ZERO;
  int4* s_meta = reinterpret_cast<int4*>(sP_ptr + 2 * TV_P_BUF);
  float* s_l = reinterpret_cast<float*>(s_meta + TV_META);
  float *s_max = s_l + TV_PTHREADS, *s_f = s_max + TV_PTHREADS;   // a tile's maxima per thread; factors of the columns' sums
  unsigned char* tail = reinterpret_cast<unsigned char*>(s_f + TV_N);
  const uint32_t bars = smem_addr(tail);
  const uint32_t full = bars, empty = full + 8 * TV_STAGES, p_full = empty + 8 * TV_STAGES, p_empty = p_full + 16, acc_done = p_empty + 16;
  uint32_t* s_tmem_base = reinterpret_cast<uint32_t*>(tail + 8 * (2 * TV_STAGES + 5));
  volatile int* abort_flag = reinterpret_cast<int*>(s_tmem_base + 1);

  const int n_pairs = (v.NC + 1) >> 1;
  uint32_t tmem_cols = 32;
  while (tmem_cols < (uint32_t)(n_pairs * TV_N)) tmem_cols <<= 1;
  if (tid == 0) {
    for (int i = 0; i < TV_STAGES; ++i) { mbar_init(full + 8 * i, 1); mbar_init(empty + 8 * i, 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(p_full + 8 * i, TV_PWARPS); mbar_init(p_empty + 8 * i, 1); }
    mbar_init(acc_done, 1);
    *abort_flag = 0;
    mbar_init_fence();
  }
  if (warp == 1) tmem_alloc(smem_addr(s_tmem_base), tmem_cols);
  for (int i = tid; i < (int)TV_ZERO / 16; i += TV_THREADS)
    reinterpret_cast<uint4*>(base_ptr + TV_STAGES * TV_STAGE)[i] = make_uint4(0u, 0u, 0u, 0u);
  fence_proxy_async_smem();
  fence_before_sync();
  __syncthreads();
  fence_after_sync();
  const uint32_t tmem_base = *s_tmem_base;

  chain_wait();
  const int4 info = a.info[req];
  const int* cut = a.vcut + (size_t)req * (a.n_splits + 1) + split;
  const int t_first = cut[0], n_mine = cut[1] - t_first;
  const int4* meta = a.vmeta + (size_t)req * (v.TPS + 1) + t_first;

  // role state that survives the descriptor chunks
  uint32_t st = 0, st_ph = 0, n_loaded = 0;                     // producer / issuer: ring stage and its phase; stages filled so far
  uint32_t touched = 0;                                         // issuer: panel pairs whose accumulator holds a value
  bool ok = true;
  int max_cls = 0;                                              // weight warps: widest class seen (which accumulators to read)
  uint64_t l_sum2 = 0;                                          // weight threads: two sums of this thread's weights
  const int pt = tid - 64, pc = pt & (TV_N - 1), tg0 = pt >> 6; // weight threads: column; token groups tg0, tg0 + 4, ...
  const bool in = c0 + pc < a.C;
  const float scale = (v.sm_scale == 0.f ? 1.f : fabsf(v.sm_scale)) * TV_LOG2E;      // scores come without their scale; weights are powers of two
  const uint64_t scale2 = tv_pack(scale, scale);
  float top = -INFINITY;                                        // weight threads: what the column's weights are relative to, times scale

  for (int k0 = 0; k0 < n_mine; k0 += TV_META) {
    const int cn = min(TV_META, n_mine - k0);
    for (int i = tid; i < cn; i += TV_THREADS) s_meta[i] = meta[k0 + i];
    __syncthreads();

    if (warp == 0) {
      // ------------------------------------------------------------- TMA producer
      if (elect_one()) {
        if (k0 == 0) { tma_prefetch_desc(&map_blocks); tma_prefetch_desc(&map_boxes); tma_prefetch_desc(&map_nodes); }
        for (int i = 0; i < cn && ok; ++i) {
          const int4 m = s_meta[i];
          const int nb = vtile_boxes(m.z);
          for (int j = 0; j < m.y; j += 2) {
            if (!(ok = mbar_wait_thin(empty + 8 * st, st_ph ^ 1u, abort_flag))) break;
            const int np = j + 1 < m.y ? 2 : 1;
            mbar_expect_tx(full + 8 * st, (uint32_t)(np * nb * JOINT_ROWS * PANEL * 2));
            for (int k = 0; k < np; ++k) {
              const uint32_t dst = sRing + st * TV_STAGE + k * TV_PANEL;
              if (m.w < 0) {
                for (int b = 0; b < nb; ++b)
                  tma_load_2d(dst + b * (JOINT_ROWS * PANEL * 2), &map_nodes, full + 8 * st, 0, (req * v.NC + j + k) * TREE_PANEL_ROWS + b * JOINT_ROWS);
              } else if (nb == TILE / JOINT_ROWS) {
                tma_load_2d(dst, &map_blocks, full + 8 * st, 0, (m.w + j + k) * TILE);
              } else {
                for (int b = 0; b < nb; ++b) tma_load_2d(dst + b * (JOINT_ROWS * PANEL * 2), &map_boxes, full + 8 * st, 0, (m.w + j + k) * TILE + b * JOINT_ROWS);
              }
            }
            ++n_loaded;
            if (++st == TV_STAGES) { st = 0; st_ph ^= 1u; }
          }
        }
        if (!ok)                                                // let copies in flight land before the CTA goes away
          for (uint32_t i = 0; i < TV_STAGES && i < n_loaded; ++i) {
            const uint32_t n = n_loaded - 1 - i;
            mbar_wait_drain(full + 8 * (n % TV_STAGES), (n / TV_STAGES) & 1u);
          }
      }
      __syncwarp();
    } else if (warp == 1) {
      // ------------------------------------------------------------- MMA issuer
      if (elect_one()) {
        constexpr uint32_t idesc = idesc_f16(BF16 ? 1 : 0, 128, TV_N) | (1u << 15);       // A MN-major, B K-major
        for (int i = 0; i < cn && ok; ++i) {
          const int k = k0 + i, cls = s_meta[i].y, nb = vtile_boxes(s_meta[i].z);
          const uint32_t buf = (uint32_t)k & 1u;
          if (!(ok = mbar_wait_thin(p_full + 8 * buf, ((uint32_t)k >> 1) & 1u, abort_flag))) break;
          const uint32_t pb = kmajor_sw128_desc_lo(sP + buf * TV_P_BUF);
          for (int j = 0; j < cls; j += 2) {
            if (!(ok = mbar_wait_thin(full + 8 * st, st_ph, abort_flag))) break;
            fence_after_sync();
            const uint32_t a0 = sRing + st * TV_STAGE;
            const bool two = j + 1 < cls;
            const uint32_t pair = (uint32_t)j >> 1, d_tmem = tmem_base + pair * TV_N;
            uint32_t acc = (touched >> pair) & 1u;
            auto step = [&](int ks) {
              const uint32_t a_addr = a0 + ks * 2048u;                                     // 16 token rows per instruction
              const uint32_t lbo = two ? TV_PANEL : sZero - a_addr;                       // where the second 64 columns are
              const uint64_t ad = ((uint64_t)KMAJOR_SW128_DESC_HI << 32) | (((a_addr >> 4) & 0x3fffu) | ((lbo >> 4) << 16));
              const uint32_t bl = pb + (ks >> 2) * (TV_P_HALF >> 4) + (ks & 3) * 2u;
              mma_f16_ss(d_tmem, ad, ((uint64_t)KMAJOR_SW128_DESC_HI << 32) | (bl + (TV_P_PART >> 4)), idesc, acc);      // low parts first
              mma_f16_ss(d_tmem, ad, ((uint64_t)KMAJOR_SW128_DESC_HI << 32) | bl, idesc, 1u);
              acc = 1u;
            };
            if (nb == TILE / JOINT_ROWS) {                      // (a loop of its own: the checks would cost this thread its pace)
#pragma unroll
              for (int ks = 0; ks < 8; ++ks) step(ks);
            } else {
#pragma unroll 1
              for (int ks = 0; ks < nb; ++ks) step(ks);
            }
            touched |= 1u << pair;
            mma_commit(empty + 8 * st);
            if (++st == TV_STAGES) { st = 0; st_ph ^= 1u; }
          }
          if (!ok) break;
          mma_commit(p_empty + 8 * buf);
        }
        if (ok && k0 + cn == n_mine) mma_commit(acc_done);
      }
      __syncwarp();
    } else {
      // ------------------------------------------------------------- weights
      // Rows that hold no token, and columns past the last, count as -inf.
      auto read = [&](int i, float (&x)[32]) {
        const int4 m = i < cn ? s_meta[i] : make_int4(0, 0, 0, 0);
        const float* p = a.scores + (size_t)m.x * TILE * a.C + c0 + pc;
#pragma unroll
        for (int it = 0; it < 4; ++it)
#pragma unroll
          for (int u = 0; u < 8; ++u) {
            const int t = (it * 4 + tg0) * 8 + u;
            x[it * 8 + u] = in && t < m.z ? p[(size_t)t * a.C] : -INFINITY;
          }
      };
      float cur[32], nxt[32];
      read(0, cur);
      for (int i = 0; i < cn; ++i) {
        const int k = k0 + i;
        const int4 m = s_meta[i];
        read(i + 1, nxt);
        // the tile's maximum of the column, from the four threads that share it
        float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int u = 0; u < 32; u += 4)
#pragma unroll
          for (int e = 0; e < 4; ++e) mx[e] = fmaxf(mx[e], cur[u + e]);
        s_max[pt] = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
        // a wait that ran out in one warp ends the loop in all of them, here: none is left at a barrier
        if (!(ok = named_bar_and(1, TV_PTHREADS, ok))) break;
        const float most = fmaxf(fmaxf(s_max[pc], s_max[pc + 64]), fmaxf(s_max[pc + 128], s_max[pc + 192])) * scale;
        const bool grow = most > top + 8.f;                       // also the first finite maximum
        const float next = grow ? most : top, f = next == top ? 1.f : tv_ex2(top - next);      // 0 where there was none yet
        top = next;
        if (tg0 == 0) s_f[pc] = f;
        float la, lb;
        tv_unpack(l_sum2, la, lb);
        l_sum2 = tv_pack(la * f, lb * f);
        if (!named_bar_and(1, TV_PTHREADS, !grow) && k > 0) {
          // seldom: what has been summed takes the factors, once the products so far have retired (those of this tile wait for its weights)
          ok = __all_sync(0xffffffffu, mbar_wait(p_empty + 8 * ((uint32_t)(k - 1) & 1u), ((uint32_t)(k - 1) >> 1) & 1u, abort_flag));
          fence_after_sync();
          const int pairs = ok ? (max_cls + 1) >> 1 : 0;
#pragma unroll 1
          for (int pair = (warp - 2) >> 2; pair < pairs; pair += 2) {
            const uint32_t at = tmem_base + ((uint32_t)((warp & 3) * 32) << 16) + (uint32_t)(pair * TV_N);
#pragma unroll 1
            for (int c = 0; c < TV_N; c += 8) {
              uint32_t o[8];
              tmem_ld8(at + c, o);
              tmem_ld_wait();
#pragma unroll
              for (int e = 0; e < 8; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * s_f[c + e]);
              tmem_st8(at + c, o);
            }
          }
          tmem_st_wait();
          fence_before_sync();
          if (!(ok = named_bar_and(1, TV_PTHREADS, ok))) break;   // the factors have been read, the sums are whole
        }
        max_cls = max(max_cls, m.y);
        const uint32_t buf = (uint32_t)k & 1u;
        ok = __all_sync(0xffffffffu, mbar_wait(p_empty + 8 * buf, (((uint32_t)k >> 1) & 1u) ^ 1u, abort_flag));
        if (!ok) continue;
        const float ref = top == -INFINITY ? 0.f : top;           // (a node that sees nothing so far has no maximum: weights stay 0)
        const uint64_t nm2 = tv_pack(-ref, -ref);
        unsigned char* pb = sP_ptr + buf * TV_P_BUF;
#pragma unroll
        for (int it = 0; it < 4; ++it) {
          const int tg = it * 4 + tg0;
          if (tg * 8 >= vtile_boxes(m.z) * JOINT_ROWS) break;        // the products leave these rows out
          uint32_t hi[4], lo[4];
#pragma unroll
          for (int u = 0; u < 8; u += 2) {
            float x0, x1;
            tv_unpack(tv_fma2(tv_pack(cur[it * 8 + u], cur[it * 8 + u + 1]), scale2, nm2), x0, x1);
            const uint64_t p = tv_pack(tv_ex2(x0), tv_ex2(x1));
            l_sum2 = tv_add2(l_sum2, p);
            split_pair_16<BF16>(p, hi[u >> 1], lo[u >> 1]);
          }
          const uint32_t off = (uint32_t)(tg >> 3) * TV_P_HALF + (uint32_t)pc * 128u + ((((uint32_t)tg & 7u) ^ ((uint32_t)pc & 7u)) << 4);
          *reinterpret_cast<uint4*>(pb + off) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
          *reinterpret_cast<uint4*>(pb + TV_P_PART + off) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_full + 8 * buf);
#pragma unroll
        for (int u = 0; u < 32; ++u) cur[u] = nxt[u];
      }
    }
    __syncthreads();                                            // the descriptors may be replaced
    ok = ok && !*abort_flag;
  }

  // ----------------------------------------------------------------- partial results of this split
  // Row of the partial results that column c of the request stands for; -1: no node's.
  auto part_row = [&](int c) -> int {
    const int g = c / a.Rs, n = c - g * a.Rs, t = n / v.rep;
    return c < a.C && n < a.R && t < info.y ? ((req * a.T + t) * a.n_splits + split) * v.Hq + g * v.rep + n % v.rep : -1;
  };
  if (warp >= 2) {
    float x, y;
    tv_unpack(l_sum2, x, y);
    s_l[pt] = x + y;
    bool ready = ok;
    if (n_mine > 0) named_bar_sync(1, TV_PTHREADS);             // the last tile's maxima have been read
    if (tg0 == 0) s_max[pc] = top;
    if (ready && n_mine > 0) ready = __all_sync(0xffffffffu, mbar_wait(acc_done, 0u, abort_flag));
    fence_after_sync();
    const int quad = warp & 3;                                  // the TMEM lanes this warp may read
    const int used_pairs = ready ? (max_cls + 1) >> 1 : 0;
    // 32 columns at a time through the ring's memory (no copy or product uses it any more) as rows of d_kv floats, each of which leaves as
    // one bulk copy.  (A split without tiles leaves its part unwritten: the merge knows it from the cut points.)
    float* s_out = reinterpret_cast<float*>(base_ptr);
    for (int n0 = 0; n0 < TV_N && c0 + n0 < a.C && n_mine > 0; n0 += TV_OUT) {
      if (n0 > 0) {
        if (warp == 2) bulk_store_wait();
        named_bar_sync(1, TV_PTHREADS);
      }
#pragma unroll 1
      for (int pair = (warp - 2) >> 2; pair < n_pairs; pair += 2) {
        const int col = pair * 128 + quad * 32 + lane;          // spectral column of this thread's TMEM lane
        const uint32_t src = tmem_base + ((uint32_t)(quad * 32) << 16) + (uint32_t)(pair * TV_N + n0);
        float val[32];
        if (pair < used_pairs) {
          tmem_ld32(src, val);
          tmem_ld_wait();
        } else {
#pragma unroll
          for (int n = 0; n < 32; ++n) val[n] = 0.f;
        }
        if (col < d_kv) {                                       // (an odd number of panels leaves half a pair)
#pragma unroll
          for (int n = 0; n < 32; ++n) s_out[n * d_kv + col] = val[n];
        }
      }
      fence_proxy_async_smem();
      named_bar_sync(1, TV_PTHREADS);
      if (warp == 2) {
        const int r = part_row(c0 + n0 + lane);
        if (r >= 0) bulk_store(a.part_acc + (size_t)r * d_kv, sRing + (uint32_t)(lane * d_kv) * 4u, (uint32_t)d_kv * 4u);
      }
    }
    if (warp == 2) bulk_store_wait();
    __syncwarp();
    tmem_ld_wait();
  }
  fence_before_sync();
  __syncthreads();
  fence_after_sync();
  if (warp == 1) tmem_dealloc(tmem_base, tmem_cols);
  if (tid < TV_N) {
    const int r = part_row(c0 + tid);
    if (r >= 0) a.part_ml[r] = make_float2(s_max[tid], (s_l[tid] + s_l[tid + 64]) + (s_l[tid + 128] + s_l[tid + 192]));
  }
  if (tid == 0 && *abort_flag) set_status(v, TWKV_ERR_TIMEOUT);
}

cudaError_t launch_tree_value(const DevView& v, const TreeCall& a, const TreeMaps& maps, cudaStream_t st) {
  ProfScope ps(TWKV_K_VACC, st);
  auto kernel = v.dtype == TWKV_BF16 ? tree_value_kernel<true> : tree_value_kernel<false>;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)TV_SMEM);
  if (e != cudaSuccess) return e;
  e = launch_chained(kernel, dim3(a.n_req * a.n_splits, (a.C + TV_N - 1) / TV_N), dim3(TV_THREADS), dim3(1), TV_SMEM, st, maps.blocks, maps.boxes, maps.node_boxes,
                     v, a);
  if (e != cudaSuccess) return e;
  count_launch();
  return cudaGetLastError();
}

}  // namespace twkv
