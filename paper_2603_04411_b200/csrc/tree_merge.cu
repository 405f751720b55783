// End of tree attention: sum of the splits, division by the sum of the weights, projection out_h = (acc_h / l_h) U_V^-1[:, head slice].
//
// A cluster of CL CTAs per (128 rows, KV head): row = (request, node; head of the group), and CTA c takes the spectral components
// [c d/CL, (c + 1) d/CL), up to 128 at a time.  It sums their splits, each relative to its own maximum, normalises, and makes them the A operand of
// a tcgen05 product with its rows of U_V^-1 (as they lie: MN-major B): two 16-bit parts of the cache type per component (three where a bf16 cache
// has fp32 outputs), fp32 accumulation in tensor memory.  The CL partial products meet in distributed shared memory, 128 / CL columns per CTA.
// What bounds it is the way of the partial sums (4 d_kv bytes per row and split) into the SMs, and for few rows the chain of reads, which a
// cluster of eight shortens; with many rows the exchange would cost more than the rest (64 KiB per CTA of eight), so CL is the largest that leaves
// two CTAs per SM.  Where a cluster of eight leaves room, its CTAs take 64 or 32 of their 128 rows (one tree of 16 nodes, 32 splits: 60 us with 128,
// 58 with 64, 42 with 32; the products' idle rows cost nothing that shows).  The decode merge does the product by FMAs, which for hundreds of nodes cost
// several times the reads (256 nodes of 32 heads 373 us by a CTA per row).
// chain_start() stands behind the allocation of tensor memory: two CTAs of this kernel share an SM, so the next kernel of the chain must
// not find columns free that one of them still needs.
#include "twkv_dev.h"
#include "tc_util.cuh"
#include "mma_util.cuh"
#include "tree.h"

namespace twkv {
using namespace tc;

constexpr int TM_THREADS = 256;
constexpr uint32_t TM_PANEL = 16384;                          // [128 rows][64 components] of one part
constexpr uint32_t TM_A = 4 * TM_PANEL, TM_B = 32768;         // two parts of up to 128 components (three of 64); their rows of U_V^-1, 128 columns
constexpr int TM_LEAST = 32;                                  // least rows of a CTA
constexpr int TM_TABLE = 4 * TILE;                            // parts whose places and weights are looked up once: four per row of 128, sixteen of 32
constexpr uint32_t TM_SMEM = TM_A + TM_B + TILE * (4 * 4 + 16) + TM_TABLE * (TREE_MAX_RANGES * 4 + 8) + 64;
static_assert(2 * TM_SMEM <= 228 * 1024 - 2 * 1024, "two CTAs per SM");
static_assert(TILE * HEAD_DIM * 4 <= TM_A, "the partial products arrive where the A operand was");

__device__ __forceinline__ float tm_ex2(float x) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }

template <bool BF16, int PARTS, int CL>
__global__ void __launch_bounds__(TM_THREADS, 2) tree_merge_kernel(const __grid_constant__ CUtensorMap map_uv, DevView v, TreeCall a) {
  extern __shared__ __align__(1024) unsigned char smem[];
  const uint32_t sA = smem_addr(smem), sB = sA + TM_A;
  float *s_most = reinterpret_cast<float*>(smem + TM_A + TM_B), *s_inv = s_most + TILE, *s_back = s_inv + TILE, *s_give = s_back + TILE;      // per row
  int4* s_row = reinterpret_cast<int4*>(s_give + TILE);                                              // first part, splits, request, row of the outputs; -1: none
  // per row and split: what its part is worth, per range of panels; the part, its components
  float4* s_w = reinterpret_cast<float4*>(s_row + TILE);
  int2* s_part = reinterpret_cast<int2*>(s_w + TM_TABLE);
  unsigned char* tail = reinterpret_cast<unsigned char*>(s_part + TM_TABLE);
  const uint32_t b_full = smem_addr(tail), done = b_full + 8;
  uint32_t* s_tmem = reinterpret_cast<uint32_t*>(tail + 16);
  volatile int* abort_flag = reinterpret_cast<int*>(s_tmem + 1);
  int* s_used = reinterpret_cast<int*>(s_tmem + 2);                                    // most splits of a row
  constexpr uint32_t PART = PARTS == 3 ? TM_PANEL : 2 * TM_PANEL;                     // bytes of one part of the A operand
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int c = CL > 1 ? (int)cluster_cta_rank() : 0, g = blockIdx.y, rep = v.rep, jn = a.m_comps;      // components at a time: a multiple of 16, at most 128
  const int slots = a.m_rows / rep, slot0 = (blockIdx.x / CL) * slots, n_slots = min(slot0 + slots, a.n_req * a.T);
  const bool misaligned = (sA & 1023u) != 0;
  if (tid == 0) {
    mbar_init(b_full, 1);
    mbar_init(done, 1);
    *abort_flag = misaligned ? 1 : 0;
    *s_used = 0;
    mbar_init_fence();
  }
  if (warp == 1) tmem_alloc(smem_addr(s_tmem), 256);
  fence_before_sync();
  __syncthreads();
  fence_after_sync();
  chain_start();
  const uint32_t tmem = *s_tmem;
  chain_wait();
  // Two to eight lanes per row (slot, h), slot = request * T + node: where its parts are, the largest reference of its splits, one over the sum of all
  // weights; and what the parts are worth, where the table holds them.  The components of a range of panels have a reference of their own; behind a
  // split's widest class there are none.  Looked up here once, so that the reads below depend on shared memory only.
  const int few = TM_TABLE / a.m_rows;
  const bool exacting = v.out_dtype == TWKV_F32, two = exacting && v.d_kv / CL > jn;    // two sums of every other chunk: long chains lose bits that fp32 outputs have
  {
    const int lanes = TM_THREADS / a.m_rows, r = tid / lanes, j = tid % lanes;
    const int slot = slot0 + r / rep, req = slot / a.T, t = slot - req * a.T;
    const int4 info = slot < n_slots ? a.info[req] : make_int4(0, 0, 0, 0);
    const bool in = slot < n_slots && t < info.y;
    const int row = in ? slot * a.n_splits * v.Hq + g * rep + r % rep : -1, used = in ? info.w : 0;      // splits that hold something come first
    float most = -INFINITY, sum = 0.f, size = 0.f;              // size: bound on the components, relative to most
    int wide = 0;                                               // widest class of the splits
    for (int s0 = j; s0 < used; s0 += 4 * lanes) {
      float4 y[4];
      float l[4];
      float4 x[4];
      int cls[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int sp = s0 + k * lanes;
        if constexpr (!BF16) x[k] = sp < used ? a.part_x[row + (size_t)sp * v.Hq] : make_float4(0.f, 0.f, 0.f, 0.f);
        y[k] = sp < used ? a.part_m[row + (size_t)sp * v.Hq] : make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
        l[k] = sp < used ? a.part_l[row + (size_t)sp * v.Hq] : 0.f;
        cls[k] = sp < used ? a.part_cls[req * a.n_splits + sp] : 0;
      }
      const float m = fmaxf(fmaxf(fmaxf(y[0].x, y[1].x), fmaxf(y[2].x, y[3].x)), most);
      sum *= most == -INFINITY ? 0.f : tm_ex2(most - m);        // (one that is not a number stays one)
      size *= most == -INFINITY ? 0.f : tm_ex2(most - m);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float w = y[k].x == -INFINITY ? 0.f : tm_ex2(y[k].x - m);
        sum += l[k] * w;
        wide = max(wide, cls[k]);
        if constexpr (!BF16) {                                   // a range's components are relative to its own reference
          const float ref[TREE_MAX_RANGES] = {y[k].x, y[k].y, y[k].z, y[k].w}, big[TREE_MAX_RANGES] = {x[k].x, x[k].y, x[k].z, x[k].w};
          float of_split = 0.f;
#pragma unroll
          for (int e = 0; e < TREE_MAX_RANGES; ++e)
            if (e * a.range < v.NC && ref[e] != -INFINITY) of_split = fmaxf(of_split, big[e] * tm_ex2(ref[e] - m));
          size += of_split;
        }
        if (s0 + k * lanes < few) s_w[r * few + s0 + k * lanes] = y[k];
      }
      most = m;
    }
    float all = most;
    for (int o = lanes / 2; o > 0; o >>= 1) all = fmaxf(all, __shfl_xor_sync(0xffffffffu, all, o));
    sum *= most == -INFINITY ? 0.f : tm_ex2(most - all);
    size *= most == -INFINITY ? 0.f : tm_ex2(most - all);
    for (int o = lanes / 2; o > 0; o >>= 1) wide = max(wide, __shfl_xor_sync(0xffffffffu, wide, o));
    for (int o = lanes / 2; o > 0; o >>= 1) { sum += __shfl_xor_sync(0xffffffffu, sum, o); size += __shfl_xor_sync(0xffffffffu, size, o); }
    float inv = sum == 0.f ? 0.f : 1.f / sum, back = 1.f;       // 0: no token seen
    if constexpr (!BF16) {
      // f16 operands: the components go up to 2^14 by a power of two, which the outputs are divided by, so that the low part of small ones keeps its bits
      const int e = (int)(__float_as_uint(size * inv) >> 23) - 127;                    // size * inv in [2^e, 2^(e + 1))
      const int up = e > -60 && e < 60 ? 13 - e : 0;
      back = __uint_as_float((unsigned)(127 - up) << 23);
      inv *= __uint_as_float((unsigned)(127 + up) << 23);
    }
    for (int k = j; k < few; k += lanes) {
      s_part[r * few + k] = k < used ? make_int2(row + k * v.Hq, a.part_cls[req * a.n_splits + k] * PANEL) : make_int2(0, 0);
      if (k >= used) continue;
      const float4 y = s_w[r * few + k];
      s_w[r * few + k] = make_float4(y.x == -INFINITY ? 0.f : tm_ex2(y.x - all) * inv, y.y == -INFINITY ? 0.f : tm_ex2(y.y - all) * inv,
                                     y.z == -INFINITY ? 0.f : tm_ex2(y.z - all) * inv, y.w == -INFINITY ? 0.f : tm_ex2(y.w - all) * inv);
    }
    if (j == 0) {
      s_row[r] = make_int4(row, used, req, in ? info.x + t : -1);
      s_most[r] = all;
      s_inv[r] = inv;
      s_back[r] = back;
      s_give[r] = (float)wide;
      if (used > 0) atomicMax(s_used, used);
    }
  }
  __syncthreads();
  // Sums: a lane takes four components of a row; a warp rows warp, warp + 8, ..., two at a time where half of its lanes are enough for one.  Eight reads on
  // their way: of as many rows where the table has the row's splits, of eight splits otherwise.  (16384 rows of one split one after the other took 204 us.)
  // What bounds it is the issue of instructions, so places and weights come from the table, and no lane is idle (37 trees of 13 nodes, fp32 outputs: 31 us
  // with a look-up per row and part and 16 idle lanes, 21 us so; 20 trees of 4 nodes, three splits: 32 and 24 us).
  const int fold = jn <= 64 ? 2 : 1, e0 = (lane & (32 / fold - 1)) * 4, its = a.m_rows / 8 / fold;
  const int r0 = warp + (fold == 2 ? (lane >> 4) * 8 : 0);         // row of iteration i: r0 + 8 fold i, so its place in a swizzled group of eight rows is warp
  const bool mine = e0 < jn;
  unsigned char* const dst0 = smem + (e0 >> 6) * TM_PANEL + r0 * 128 + ((((e0 >> 3) & 7) ^ warp) << 4) + (e0 & 7) * 2;
  uint32_t seconds = 0u;                                       // rows (by iteration) that have a second part somewhere
  auto put = [&](int i, float4 x) {                             // a row's normalised components as the A operand
    if (!mine) return;
    uint32_t w[PARTS][2];                                       // the largest part first
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint64_t y;
      asm("mov.b64 %0, {%1, %2};" : "=l"(y) : "f"(h ? x.z : x.x), "f"(h ? x.w : x.y));
      if constexpr (PARTS == 3) tree_split3(y, w[0][h], w[1][h], w[2][h]);
      else split_pair_16<BF16>(y, w[0][h], w[1][h]);
    }
#pragma unroll
    for (int p = 0; p < PARTS; ++p) *reinterpret_cast<uint2*>(dst0 + p * PART + i * fold * 1024) = make_uint2(w[p][0], w[p][1]);
    if (exacting && (w[1][0] | w[1][1]) != 0u) seconds |= 1u << i;
  };
  const int used = *s_used;
  bool ok = !misaligned;
  uint32_t ph = 0;
  const int first = c * (v.d_kv / CL), n_chunks = v.d_kv / CL / jn;
  for (int chunk = 0; chunk < n_chunks; ++chunk) {
    const int j0 = first + chunk * jn, comp = j0 + e0, range = comp / (a.range * PANEL);
    if (warp == 0 && elect_one() && ok) {                      // U_V^-1, on its way while the splits are summed
      mbar_expect_tx(b_full, (uint32_t)jn * 256u);
      tma_load_2d(sB, &map_uv, b_full, g * HEAD_DIM, j0);
      tma_load_2d(sB + jn * 128u, &map_uv, b_full, g * HEAD_DIM + 64, j0);
    }
    __syncwarp();
    const float* const acc = a.part_acc + comp;
    if (used <= few) {
      const float* const s_wr = reinterpret_cast<const float*>(s_w) + range;
#pragma unroll 1
      for (int i0 = 0; i0 < its; i0 += 8) {
        float4 x[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = make_float4(0.f, 0.f, 0.f, 0.f);
        const int at = (r0 + 8 * fold * i0) * few;
#pragma unroll 1
        for (int s = 0; s < used; ++s) {
          float4 y[8];
          float w[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            y[k] = make_float4(0.f, 0.f, 0.f, 0.f);
            w[k] = 0.f;
            if (i0 + k < its) {
              const int n = at + 8 * fold * k * few + s;
              const int2 part = s_part[n];
              if (mine && comp < part.y) {
                y[k] = *reinterpret_cast<const float4*>(acc + (size_t)part.x * v.d_kv);
                w[k] = s_wr[4 * n];
              }
            }
          }
#pragma unroll
          for (int k = 0; k < 8; ++k) { x[k].x += y[k].x * w[k]; x[k].y += y[k].y * w[k]; x[k].z += y[k].z * w[k]; x[k].w += y[k].w * w[k]; }
        }
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (i0 + k < its) put(i0 + k, x[k]);
      }
    } else {
#pragma unroll 1
      for (int i = 0; i < its; ++i) {
        const int r = r0 + 8 * fold * i;
        const int4 q = s_row[r];                                  // (no row: no splits)
        const int* cls = a.part_cls + q.z * a.n_splits;
        const float* refs = reinterpret_cast<const float*>(a.part_m + max(q.x, 0)) + range;
        const float most = s_most[r], inv = s_inv[r];
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
        for (int s0 = 0; s0 < q.y; s0 += 8) {
          float4 y[8];
          float ref[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const bool in = mine && s0 + k < q.y && comp < cls[s0 + k] * PANEL;
            y[k] = in ? *reinterpret_cast<const float4*>(acc + (size_t)(q.x + (s0 + k) * v.Hq) * v.d_kv) : make_float4(0.f, 0.f, 0.f, 0.f);
            ref[k] = in ? refs[(size_t)(s0 + k) * v.Hq * 4] : -INFINITY;
          }
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const float w = ref[k] == -INFINITY ? 0.f : tm_ex2(ref[k] - most);
            x.x += y[k].x * w; x.y += y[k].y * w; x.z += y[k].z * w; x.w += y[k].w * w;
          }
        }
        put(i, make_float4(x.x * inv, x.y * inv, x.z * inv, x.w * inv));
      }
    }
    fence_proxy_async_smem();
    __syncthreads();
    if (warp == 0 && elect_one() && ok) {
      if (mbar_wait(b_full, ph, abort_flag)) {
        fence_after_sync();
        constexpr uint32_t idesc = idesc_f16(BF16 ? 1 : 0, 128, 128) | (1u << 16);       // B MN-major
        const uint32_t d = tmem + (two ? (uint32_t)(chunk & 1) * 128u : 0u);
        const uint32_t b_lo = ((sB >> 4) & 0x3fffu) | ((uint32_t)(jn * 128) >> 4 << 16);
        for (int part = PARTS - 1; part >= 0; --part)                     // the low parts first: the sum is cut after every instruction
          for (int ks = 0; ks < jn / 16; ++ks) {
            const uint32_t a_lo = kmajor_sw128_desc_lo(sA + part * PART + (ks >> 2) * TM_PANEL) + 2 * (ks & 3);
            mma_f16_ss(d, ((uint64_t)KMAJOR_SW128_DESC_HI << 32) | a_lo, ((uint64_t)KMAJOR_SW128_DESC_HI << 32) | (b_lo + ks * 128u), idesc,
                       chunk > (two ? 1 : 0) || part < PARTS - 1 || ks > 0 ? 1u : 0u);
          }
        mma_commit(done);
      }
    }
    __syncwarp();
    ok = ok && __all_sync(0xffffffffu, mbar_wait(done, ph, abort_flag));      // (the operands may be replaced)
    ph ^= 1u;
    fence_after_sync();
    __syncthreads();
  }
  if (exacting) {
    // fp32 outputs get back what the sums of the products are expected to lose (16-bit ones would not show it), by the instructions that had components
    // (none behind the row's widest class): each of the first part, and of the others where the row has any (means of one token have none); those of
    // bf16's two others count once the sum has its size, f16's, whose products are longer, at once.  Every lane of a row has seen its own components.
    for (int o = 16 / fold; o > 0; o >>= 1) seconds |= __shfl_xor_sync(0xffffffffu, seconds, o);
    const int i = lane & (32 / fold - 1);
    if (i < its) {
      const int r = r0 + 8 * fold * i, n = min(max((int)s_give[r] * PANEL - first, 0), v.d_kv / CL) / 16;
      const int rest = PARTS == 3 ? 2 * max(n - (two ? 2 : 1) * jn / 16, 0) : n;
      s_give[r] = 1.f + TREE_CUT * (two ? 0.5f : 1.f) * (float)(n + ((seconds >> i) & 1u ? rest : 0));
    }
    __syncthreads();
  }
  constexpr int CW = HEAD_DIM / CL;                             // columns a CTA writes
  if constexpr (CL > 1) cluster_sync_all();                     // every CTA's A operand has been used: the parts may arrive there
  if ((warp & 3) * 32 < a.m_rows) {
    const int quarter = warp & 3, half = warp >> 2, row = quarter * 32 + lane;
    const float give = s_give[row];
    float x[32];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int col = half * 64 + k * 32;
      if (ok) {
        tmem_ld32(tmem + ((uint32_t)(quarter * 32) << 16) + col, x);
        tmem_ld_wait();
        if (two) {
          float y[32];
          tmem_ld32(tmem + ((uint32_t)(quarter * 32) << 16) + 128 + col, y);
          tmem_ld_wait();
#pragma unroll
          for (int e = 0; e < 32; ++e) x[e] += y[e];
        }
        if (exacting) {
#pragma unroll
          for (int e = 0; e < 32; ++e) x[e] *= give;
        }
      } else {
#pragma unroll
        for (int e = 0; e < 32; ++e) x[e] = 0.f;
      }
      // four columns to the CTA that writes them: [from][four columns][row], so that a warp's rows lie together
#pragma unroll
      for (int e = 0; e < 32; e += 4) {
        const uint32_t at = sA + (uint32_t)(((c * CW + (col + e) % CW) / 4 * TILE + row) * 16);
        const float4 w = make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]);
        if constexpr (CL > 1) st_cluster_f32x4(cluster_map(at, (uint32_t)((col + e) / CW)), w);
        else *reinterpret_cast<float4*>(smem + (at - sA)) = w;
      }
    }
  }
  fence_before_sync();
  if constexpr (CL > 1) cluster_sync_all();                     // every part has arrived; nothing remote is touched from here on
  else __syncthreads();
  fence_after_sync();
  if (warp == 1) tmem_dealloc(tmem, 256);
  {
    const int r = tid & (TILE - 1), e0 = (tid >> 7) * (CW / 2);
    const int4 q = r < a.m_rows ? s_row[r] : make_int4(0, 0, 0, -1);
    if (q.w >= 0) {
      const bool bad = q.y > 0 && (a.masks[q.w] & a.bad[q.z]);    // sees a node whose value is not finite
#pragma unroll 2
      for (int e1 = e0; e1 < e0 + CW / 2; e1 += 8) {
        float o[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = 0.f;
#pragma unroll
        for (int k = 0; k < CL; ++k) {                            // fixed order
          const float4* in = reinterpret_cast<const float4*>(smem) + (k * CW + e1) / 4 * TILE + r;
          const float4 x = in[0], y = in[TILE];
          o[0] += x.x; o[1] += x.y; o[2] += x.z; o[3] += x.w; o[4] += y.x; o[5] += y.y; o[6] += y.z; o[7] += y.w;
        }
        if constexpr (!BF16) {
          const float back = s_back[r];
#pragma unroll
          for (int e = 0; e < 8; ++e) o[e] *= back;
        }
        if (bad) {
#pragma unroll
          for (int e = 0; e < 8; ++e) o[e] = __int_as_float(0x7fffffff);
        }
        const size_t at = ((size_t)q.w * v.Hq + g * rep + r % rep) * HEAD_DIM + c * CW + e1;
        if (v.out_dtype == TWKV_F32) {
          float4* d = reinterpret_cast<float4*>(reinterpret_cast<float*>(a.out) + at);
          d[0] = make_float4(o[0], o[1], o[2], o[3]);
          d[1] = make_float4(o[4], o[5], o[6], o[7]);
        } else {
          unsigned w[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            if (v.out_dtype == TWKV_BF16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[k]) : "f"(o[2 * k + 1]), "f"(o[2 * k]));
            else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(w[k]) : "f"(o[2 * k + 1]), "f"(o[2 * k]));
          }
          *reinterpret_cast<uint4*>(reinterpret_cast<unsigned short*>(a.out) + at) = make_uint4(w[0], w[1], w[2], w[3]);
        }
      }
    }
  }
  if (tid == 0 && *abort_flag) set_status(v, misaligned ? TWKV_ERR_DEVICE_CHECK : TWKV_ERR_TIMEOUT);
}

// CTAs of a cluster, and rows that one takes: as many and as few as leave two CTAs per SM.
int tree_merge_cluster(const DevView& v, const TreeCall& a, int sm_count, int* rows) {
  auto tiles = [&](int rows) { return (a.n_req * a.T + rows / v.rep - 1) / (rows / v.rep) * v.Hkv; };
  int cl = 8;
  while (cl > 1 && tiles(TILE) * cl > 2 * sm_count) cl /= 2;
  *rows = TILE;
  while (*rows > TM_LEAST && *rows / 2 >= v.rep && tiles(*rows / 2) * cl <= 2 * sm_count) *rows /= 2;
  return cl;
}
// Components that a CTA takes at a time: the least number of equal pieces of at most 128 (three parts: 64), a multiple of sixteen each.
int tree_merge_comps(int d_kv, int cl, int parts) {
  const int most = parts == 3 ? 64 : 128;
  int n = (d_kv / cl + most - 1) / most;
  while (d_kv / cl % (16 * n)) ++n;
  return d_kv / cl / n;
}

template <bool BF16, int PARTS, int CL>
static cudaError_t launch_tree_merge_t(const DevView& v, const TreeCall& a, const TreeMaps& maps, cudaStream_t st) {
  cudaError_t e = cudaFuncSetAttribute(tree_merge_kernel<BF16, PARTS, CL>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)TM_SMEM);
  if (e != cudaSuccess) return e;
  const int slots = a.m_rows / v.rep, tiles = (a.n_req * a.T + slots - 1) / slots;
  return launch_chained(tree_merge_kernel<BF16, PARTS, CL>, dim3(CL * tiles, v.Hkv), dim3(TM_THREADS), dim3(CL), TM_SMEM, st, maps.uv, v, a);
}
template <bool BF16, int PARTS>
static cudaError_t launch_tree_merge_cl(const DevView& v, const TreeCall& a, const TreeMaps& maps, cudaStream_t st) {
  switch (a.m_cluster) {
    case 1: return launch_tree_merge_t<BF16, PARTS, 1>(v, a, maps, st);
    case 2: return launch_tree_merge_t<BF16, PARTS, 2>(v, a, maps, st);
    case 4: return launch_tree_merge_t<BF16, PARTS, 4>(v, a, maps, st);
    default: return launch_tree_merge_t<BF16, PARTS, 8>(v, a, maps, st);
  }
}
cudaError_t launch_tree_merge(const DevView& v, const TreeCall& a, const TreeMaps& maps, cudaStream_t st) {
  ProfScope ps(TWKV_K_MERGE, st);
  const cudaError_t e = v.dtype != TWKV_BF16 ? launch_tree_merge_cl<false, 2>(v, a, maps, st)
                      : a.n_parts == 3 ? launch_tree_merge_cl<true, 3>(v, a, maps, st) : launch_tree_merge_cl<true, 2>(v, a, maps, st);
  if (e != cudaSuccess) return e;
  count_launch();
  return cudaGetLastError();
}

}  // namespace twkv
