// Scores of drafted trees on the 5th-generation tensor cores.
//
// Per K tile (128 tokens, c panels) and KV head g, as in a decode pass (kscore_tc.cu):
//   Kbar_g = X^_K U_K^-1[:, g]  (Eq. 3),  Krot_g = RoPE(Kbar_g),  S_g = Krot_g Q_g^T
// with all query rows of the request, nodes x heads of the group, in Q_g.  A tile is rebuilt and rotated once for all of them; that is
// what a pass of single queries per node repeats.  The kernel runs on CTA pairs (M = 256 over two tiles of ONE request, so that
// each CTA holds half of Q_g's rows and every column of the product is wanted).  Query rows go through in blocks of 64 columns
// (N = 16 .. 64): their operand, made by the plan kernel, streams through a ring of three stages, a block's scores land in one of two
// accumulators and leave through shared memory, so that a token's scores are stored as whole lines.
//
// Tensor memory (512 columns): slabs of rebuilt keys 3 x 128 | score accumulators 2 x 64.
// Warp roles (512 threads, one persistent CTA per SM; registers re-divided by warpgroup):
//   warp 0      TMA producer of U_K^-1 panels
//   warp 1      issuer of the reconstruction products (even CTA; owns the TMEM allocation)
//   warp 2      TMA producer of X^_K panels
//   warp 3      issuer of the score products (even CTA), and in both CTAs the producer of the query blocks, two ahead
//   warps 4-11  rotation and high / low split (thread = one token row x half of the RoPE frequencies)
//   warps 12-15 scores out: scaled, masked (nodes), transposed through shared memory, stored, folded into the running maxima
// A class wider than eight panels runs as two passes over its panels, the second adding to the scores the first one stored.
// All waits are bounded (tc_util.cuh); a wait that runs out ends the kernel with TWKV_ERR_TIMEOUT.
#include "twkv_dev.h"
#include "tc_util.cuh"
#include "tree.h"

namespace twkv {
using namespace tc;

constexpr int TS_THREADS = 512;
constexpr int TS_REGS_LIGHT = 56, TS_REGS_EPI = 184, TS_REGS_OUT = 80;      // 128 x 56 + 256 x 184 + 128 x 80 = 64512 of 65536
constexpr int TS_A_SLOTS = 8, TS_B_STAGES = 3, TS_Q_STAGES = 3, TS_SLABS = 3, TS_S_SLOTS = 2;
constexpr uint32_t TS_PANEL = 16384, TS_B_PART = 8192, TS_B_STAGE = 2 * TS_B_PART;
constexpr int TS_QCOLS = 64;                                    // query rows of a block, half of them in each CTA
constexpr uint32_t TS_Q_PANEL = TS_QCOLS / 2 * 128, TS_Q_STAGE = 2 * TS_Q_PANEL;
constexpr uint32_t TS_COL_SLAB = 0, TS_COL_S = 128 * TS_SLABS;
constexpr int TS_ROPE_STRIDE = 33;                              // float4 per row of the small RoPE table (32 + 1 against bank conflicts)
constexpr uint32_t TS_ROPE_BYTES = ROPE_LO * TS_ROPE_STRIDE * 16;
constexpr uint32_t TS_OUT_WARP = 32 * 128;                      // 32 token rows x 32 columns of a warp on their way out
constexpr int TS_N_BARS = 2 * TS_A_SLOTS + 2 * TS_B_STAGES + 2 * TS_Q_STAGES + 3 * TS_SLABS + 2 * TS_S_SLOTS;
constexpr uint32_t TS_SMEM = TS_A_SLOTS * TS_PANEL + TS_B_STAGES * TS_B_STAGE + TS_Q_STAGES * TS_Q_STAGE + 4 * TS_OUT_WARP + TS_ROPE_BYTES + 8 * TS_N_BARS + 16;
static_assert(TS_SMEM > CHAIN_TMEM_SMEM && TS_SMEM <= 232448, "no other CTA with tensor memory beside this one");
static_assert(TS_COL_S + TS_QCOLS * TS_S_SLOTS <= 512, "tensor memory");

__device__ __forceinline__ uint64_t ts_pack(float a, float b) { uint64_t r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ uint64_t ts_pack_bits(uint32_t a, uint32_t b) { uint64_t r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "r"(a), "r"(b)); return r; }
__device__ __forceinline__ uint64_t ts_mul(uint64_t a, uint64_t b) { uint64_t r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ uint64_t ts_sub(uint64_t a, uint64_t b) { uint64_t r; asm("sub.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ uint64_t ts_fma(uint64_t a, uint64_t b, uint64_t c) { uint64_t r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }

// A work unit: this CTA's list entry, and the class of the pair (that of its wider tile, the even CTA's).
struct TsUnit {
  int4 e;
  int cls;
};

template <bool BF16, bool DBG>
__global__ void __launch_bounds__(TS_THREADS, 1)
tree_score_kernel(const __grid_constant__ CUtensorMap map_blocks, const __grid_constant__ CUtensorMap map_boxes, const __grid_constant__ CUtensorMap map_nodes,
                  const __grid_constant__ CUtensorMap map_uinvT, const __grid_constant__ CUtensorMap map_q, DevView v, TreeCall a, int layer) {
  chain_start();
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t crank = cluster_cta_rank();
  const uint32_t sA = smem_addr(smem_raw);
  const bool misaligned = (sA & 1023u) != 0;
  const uint32_t sB = sA + TS_A_SLOTS * TS_PANEL, sQ = sB + TS_B_STAGES * TS_B_STAGE;
  unsigned char* out_stage = smem_raw + TS_A_SLOTS * TS_PANEL + TS_B_STAGES * TS_B_STAGE + TS_Q_STAGES * TS_Q_STAGE;
  float4* sRope = reinterpret_cast<float4*>(out_stage + 4 * TS_OUT_WARP);
  unsigned char* tail = out_stage + 4 * TS_OUT_WARP + TS_ROPE_BYTES;
  const uint32_t bars = smem_addr(tail);
  // In the even CTA, also for the odd one's copies and arrivals: a_full, b_full, q_full, kr_full, slab_empty, s_empty.  In both, signalled
  // together by a multicast commit: a_empty, b_empty, q_empty, slab_full, s_full.
  const uint32_t a_full = bars, a_empty = a_full + 8 * TS_A_SLOTS, b_full = a_empty + 8 * TS_A_SLOTS, b_empty = b_full + 8 * TS_B_STAGES;
  const uint32_t q_full = b_empty + 8 * TS_B_STAGES, q_empty = q_full + 8 * TS_Q_STAGES, slab_full = q_empty + 8 * TS_Q_STAGES;
  const uint32_t kr_full = slab_full + 8 * TS_SLABS, slab_empty = kr_full + 8 * TS_SLABS, s_full = slab_empty + 8 * TS_SLABS, s_empty = s_full + 8 * TS_S_SLOTS;
  uint32_t* s_tmem_base = reinterpret_cast<uint32_t*>(tail + 8 * TS_N_BARS);
  volatile int* abort_flag = reinterpret_cast<int*>(s_tmem_base + 1);
  const uint32_t a_full_even = cluster_map(a_full, 0), b_full_even = cluster_map(b_full, 0), q_full_even = cluster_map(q_full, 0);
  const uint32_t kr_full_even = cluster_map(kr_full, 0), s_empty_even = cluster_map(s_empty, 0);

  if (tid == 0) {
    for (int i = 0; i < TS_A_SLOTS; ++i) { mbar_init(a_full + 8 * i, 1); mbar_init(a_empty + 8 * i, 1); }
    for (int i = 0; i < TS_B_STAGES; ++i) { mbar_init(b_full + 8 * i, 1); mbar_init(b_empty + 8 * i, 1); }
    for (int i = 0; i < TS_Q_STAGES; ++i) { mbar_init(q_full + 8 * i, 1); mbar_init(q_empty + 8 * i, 1); }
    for (int i = 0; i < TS_SLABS; ++i) { mbar_init(slab_full + 8 * i, 1); mbar_init(kr_full + 8 * i, 2 * 8); mbar_init(slab_empty + 8 * i, 1); }
    for (int i = 0; i < TS_S_SLOTS; ++i) { mbar_init(s_full + 8 * i, 1); mbar_init(s_empty + 8 * i, 2 * 4); }
    *abort_flag = misaligned ? 1 : 0;
    mbar_init_fence();
  }
  if (warp == 1) tmem_alloc_pair(smem_addr(s_tmem_base), 512);
  chain_wait();
  for (int i = tid; i < ROPE_LO * 32; i += TS_THREADS) sRope[(i >> 5) * TS_ROPE_STRIDE + (i & 31)] = v.rope_lo[i];
  fence_before_sync();
  __syncthreads();
  cluster_sync_all();                                           // both CTAs' barriers and TMEM are ready
  fence_after_sync();
  const uint32_t tmem_base = *s_tmem_base;

  // this pair's contiguous piece [w0, total) of the list's item parts, cut by estimated cost; a part is nh of the KV heads of an item
  const int piece = (int)(blockIdx.x >> 1);
  const int w0 = a.cta_start[piece], total = a.cta_start[piece + 1];
  const int hs = __ffs(*a.parts) - 1, nh = v.Hkv >> hs;
  const int n_sub = (a.Rp + TS_QCOLS - 1) / TS_QCOLS;
  auto unit = [&](int w) -> TsUnit {
    TsUnit u;
    if (w < total) {
      const int4* p = a.klist + 2 * (size_t)(w >> hs);
      u.e = p[crank];
      u.cls = p[0].y & TREE_CLASS;
    } else {
      u.e = make_int4(0, 0, 0, -1);
      u.cls = 0;
    }
    return u;
  };
  // K slot of a row of an entry in the cache, -1 where it holds no token
  auto cache_slot = [&](const int4& e, int row) -> int {
    if (e.x < 0) return v.joint_rows()[(size_t)~e.x * TILE + row];
    return row < (e.y >> 16) ? e.x * TILE + row : -1;
  };
  auto cached = [](const int4& e) -> bool { return e.w >= 0 && (e.y & (TREE_NODES | TREE_FILLER)) == 0; };
  // pairs walk the KV heads in rotated order, so that at any moment they read different panels of U_K^-1 from L2
  const int g_rot = piece % nh;
  auto first_head = [&](int w) -> int { return (w & ((1 << hs) - 1)) * nh; };
  auto head = [&](int g0, int sl) -> int { return g0 + (sl + g_rot < nh ? sl + g_rot : sl + g_rot - nh); };

  if (misaligned) {
    // nothing was started; fall through to the common exit
  } else if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(TS_REGS_LIGHT));
    if (warp == 2) {
      // ----------------------------------------------------------- TMA producer: X^_K panels
      if (elect_one()) {
        tma_prefetch_desc(&map_blocks);
        tma_prefetch_desc(&map_boxes);
        tma_prefetch_desc(&map_nodes);
        uint32_t ak = 0;                                        // panels so far; slot = ak % 8
        bool ok = true;
        TsUnit u = unit(w0);
        for (int w = w0; w < total && ok; ++w) {
          const TsUnit nxt = unit(w + 1);
          const int own = u.e.y & TREE_CLASS;
          const bool joint = u.e.x < 0, node = (u.e.y & TREE_NODES) != 0;
          unsigned box[TILE / JOINT_ROWS];
          if (joint) {
            const uint4* b4 = reinterpret_cast<const uint4*>(v.joint_boxes() + (size_t)~u.e.x * (TILE / JOINT_ROWS));
            const uint4 lo = b4[0], hi = b4[1];
            box[0] = lo.x; box[1] = lo.y; box[2] = lo.z; box[3] = lo.w; box[4] = hi.x; box[5] = hi.y; box[6] = hi.z; box[7] = hi.w;
          }
          for (int j = 0; j < u.cls; ++j, ++ak) {
            const uint32_t slot = ak % TS_A_SLOTS, ph = (ak / TS_A_SLOTS) & 1u, dst = sA + slot * TS_PANEL;
            if (!(ok = mbar_wait_thin(a_empty + 8 * slot, ph ^ 1u, abort_flag))) break;
            if (crank == 0) mbar_expect_tx(a_full + 8 * slot, 2 * TS_PANEL);            // this CTA's copy and the partner's
            if (joint) {
#pragma unroll
              for (int b = 0; b < TILE / JOINT_ROWS; ++b)       // a box of a narrower class lies behind the last block from its class on and reads zeros there
                tma_load_2d_pair(dst + b * (JOINT_ROWS * PANEL * 2), &map_boxes, a_full_even + 8 * slot, 0,
                                 j < (int)(box[b] & 31u) ? (int)(box[b] >> 5) * JOINT_ROWS + j * TILE : v.n_blocks * TILE);
            } else if (node && j < own) {
              tma_load_2d_pair(dst, &map_nodes, a_full_even + 8 * slot, 0, u.e.z + j * TREE_PANEL_ROWS);       // rows past the nodes': other panels, dropped
            } else {
              tma_load_2d_pair(dst, &map_blocks, a_full_even + 8 * slot, 0, j < own ? (u.e.z + j) * TILE : v.n_blocks * TILE);
            }
          }
          u = nxt;
        }
      }
      __syncwarp();
    } else if (warp == 0) {
      // ----------------------------------------------------------- TMA producer: U_K^-1 panels, this CTA's half of each
      if (elect_one()) {
        tma_prefetch_desc(&map_uinvT);
        uint32_t bst = 0, bph = 0;
        bool ok = true;
        TsUnit u = unit(w0);
        for (int w = w0; w < total && ok; ++w) {
          const TsUnit nxt = unit(w + 1);
          const int g0 = first_head(w);
          for (int p0 = 0; p0 < u.cls && ok; p0 += TS_A_SLOTS) {
            const int np = min(TS_A_SLOTS, u.cls - p0);
            for (int sl = 0; sl < nh && ok; ++sl) {
              const int g = head(g0, sl);
              for (int j = 0; j < np; j += 2) {
                if (!(ok = mbar_wait_thin(b_empty + 8 * bst, bph ^ 1u, abort_flag))) break;
                const int npan = min(2, np - j);
                if (crank == 0) mbar_expect_tx(b_full + 8 * bst, 2 * npan * TS_B_PART);
                for (int k = 0; k < npan; ++k)
                  tma_load_2d_pair(sB + bst * TS_B_STAGE + k * TS_B_PART, &map_uinvT, b_full_even + 8 * bst, 0,
                                   ((p0 + j + k) * v.Hkv + g) * HEAD_DIM + (int)crank * (HEAD_DIM / 2));
                if (++bst == TS_B_STAGES) { bst = 0; bph ^= 1u; }
              }
            }
          }
          u = nxt;
        }
      }
      __syncwarp();
    } else if (warp == 1) {
      // ----------------------------------------------------------- issuer of the reconstruction products
      if (crank == 0 && elect_one()) {
        const uint32_t idesc_main = idesc_f16(BF16 ? 1 : 0, 256, 128);
        const uint32_t a_lo0 = kmajor_sw128_desc_lo(sA), b_lo0 = kmajor_sw128_desc_lo(sB);
        uint32_t bst = 0, bph = 0, ak = 0, sbuf = 0, sph = 0;
        bool ok = true;
        TsUnit u = unit(w0);
        for (int w = w0; w < total && ok; ++w) {
          const TsUnit nxt = unit(w + 1);
          for (int p0 = 0; p0 < u.cls && ok; p0 += TS_A_SLOTS) {
            const int np = min(TS_A_SLOTS, u.cls - p0);
            for (int sl = 0; sl < nh && ok; ++sl) {
              // the buffer is free once the score products over its previous contents have retired
              if (!(ok = mbar_wait_thin(slab_empty + 8 * sbuf, sph ^ 1u, abort_flag))) break;
              fence_after_sync();
              const uint32_t d = tmem_base + TS_COL_SLAB + sbuf * 128;
              const bool first = sl == 0, last = sl == nh - 1;
              uint32_t an = ak;
              for (int j = 0; j < np; j += 2, an += 2) {
                const bool two = j + 1 < np;
                const uint32_t slot = an & (TS_A_SLOTS - 1), slot2 = (an + 1) & (TS_A_SLOTS - 1);
                if (first) {
                  if (!(ok = mbar_wait_thin(a_full + 8 * slot, (an >> 3) & 1u, abort_flag))) break;
                  if (two && !(ok = mbar_wait_thin(a_full + 8 * slot2, ((an + 1) >> 3) & 1u, abort_flag))) break;
                }
                const uint32_t st = bst;
                if (!(ok = mbar_wait_thin(b_full + 8 * st, bph, abort_flag))) break;
                if (++bst == TS_B_STAGES) { bst = 0; bph ^= 1u; }
                fence_after_sync();
                mma_f16_ss_panel_cg<2>(d, a_lo0 + slot * (TS_PANEL >> 4), b_lo0 + st * (TS_B_STAGE >> 4), idesc_main, j > 0 ? 1u : 0u);
                if (two) mma_f16_ss_panel_cg<2>(d, a_lo0 + slot2 * (TS_PANEL >> 4), b_lo0 + st * (TS_B_STAGE >> 4) + (TS_B_PART >> 4), idesc_main, 1u);
                mma_commit_pair_both(b_empty + 8 * st);
                if (last) { mma_commit_pair_both(a_empty + 8 * slot); if (two) mma_commit_pair_both(a_empty + 8 * slot2); }
              }
              if (!ok) break;
              mma_commit_pair_both(slab_full + 8 * sbuf);
              if (++sbuf == TS_SLABS) { sbuf = 0; sph ^= 1u; }
            }
            ak += np;
          }
          u = nxt;
        }
      }
      __syncwarp();
    } else {
      // ----------------------------------------------------------- query blocks in, score products
      if (elect_one()) {
        tma_prefetch_desc(&map_q);
        bool ok = true;
        // The blocks in order: (unit, pass, KV head, block of 64 rows).  Block n takes ring stage n % 3 once the products of block n - 3 have retired.
        int lw = w0, lp = 0, lsl = 0, lsub = 0;
        uint32_t lst = 0, lph = 0;
        TsUnit lu = unit(w0);
        auto load = [&]() -> bool {                             // the next block; nothing once all are loaded
          if (lw >= total) return true;
          if (!mbar_wait_thin(q_empty + 8 * lst, lph ^ 1u, abort_flag)) return false;
          const int half = min(TS_QCOLS, a.Rp - lsub * TS_QCOLS) / 2;
          const int y = (lu.e.w * v.Hkv + head(first_head(lw), lsl)) * a.Rp + lsub * TS_QCOLS + (int)crank * half;
          if (crank == 0) mbar_expect_tx(q_full + 8 * lst, 2 * 2 * (uint32_t)a.q_box * 128u);
          tma_load_2d_pair(sQ + lst * TS_Q_STAGE, &map_q, q_full_even + 8 * lst, 0, y);
          tma_load_2d_pair(sQ + lst * TS_Q_STAGE + TS_Q_PANEL, &map_q, q_full_even + 8 * lst, PANEL, y);
          if (++lst == TS_Q_STAGES) { lst = 0; lph ^= 1u; }
          if (++lsub == n_sub) {
            lsub = 0;
            if (++lsl == nh) {
              lsl = 0;
              lp += TS_A_SLOTS;
              if (lp >= lu.cls) { lp = 0; lu = unit(++lw); }
            }
          }
          return true;
        };
        if (crank != 0) {
          while (ok && lw < total) ok = load();
        } else {
          ok = load() && load();
          const uint32_t q_lo0 = kmajor_sw128_desc_lo(sQ);
          uint32_t sbuf = 0, sph = 0, slot = 0, slph = 0, qst = 0, qph = 0;
          TsUnit u = unit(w0);
          for (int w = w0; w < total && ok; ++w) {
            const TsUnit nxt = unit(w + 1);
            for (int p0 = 0; p0 < u.cls && ok; p0 += TS_A_SLOTS) {
              for (int sl = 0; sl < nh && ok; ++sl) {
                if (!(ok = mbar_wait_thin(kr_full + 8 * sbuf, sph, abort_flag))) break;
                const uint32_t kr = tmem_base + TS_COL_SLAB + sbuf * 128;
                for (int sub = 0; sub < n_sub; ++sub) {
                  if (!(ok = mbar_wait_thin(s_empty + 8 * slot, slph ^ 1u, abort_flag))) break;
                  if (!(ok = mbar_wait_thin(q_full + 8 * qst, qph, abort_flag))) break;
                  fence_after_sync();
                  const uint32_t idesc_s = idesc_f16(0, 256, min(TS_QCOLS, a.Rp - sub * TS_QCOLS));
                  const uint32_t sd = tmem_base + TS_COL_S + TS_QCOLS * slot, ql = q_lo0 + qst * (TS_Q_STAGE >> 4);
                  // high and low f16 parts of the rotated keys into the same accumulator, the low one first
                  mma_f16_ts_k128_cg<2>(sd, kr + 64, ql, TS_Q_PANEL >> 4, idesc_s, 0u);
                  mma_f16_ts_k128_cg<2>(sd, kr, ql, TS_Q_PANEL >> 4, idesc_s, 1u);
                  mma_commit_pair_both(q_empty + 8 * qst);
                  if (sub == n_sub - 1) mma_commit_pair(slab_empty + 8 * sbuf);
                  mma_commit_pair_both(s_full + 8 * slot);
                  if (++slot == TS_S_SLOTS) { slot = 0; slph ^= 1u; }
                  if (++qst == TS_Q_STAGES) { qst = 0; qph ^= 1u; }
                  if (!(ok = load())) break;
                }
                if (++sbuf == TS_SLABS) { sbuf = 0; sph ^= 1u; }
              }
            }
            u = nxt;
          }
        }
      }
      __syncwarp();
    }
  } else if (warp <= 11) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(TS_REGS_EPI));
    // ------------------------------------------------------------- rotation
    const int quarter = warp & 3, hf = (warp - 4) >> 2;
    const int row = quarter * 32 + lane;
    const uint32_t lane_addr = tmem_base + ((uint32_t)(quarter * 32) << 16);
    const int* kpos = v.aux(layer, 0);
    const float4* __restrict__ rope_hi = v.rope_hi;
    uint32_t sbuf = 0, sph = 0;
    bool ok = true;
    uint64_t cs2[16], sn2[16];                                    // the tile's rotation factors, frequencies (2 t, 2 t + 1) packed
    auto rope_setup = [&](int pos) {
      const float4* __restrict__ th = rope_hi + (size_t)((pos >> 4) & (ROPE_HI - 1)) * 32 + hf * 16;
      const float4* tl = sRope + (pos & 15) * TS_ROPE_STRIDE + hf * 16;
      float4 h[16];
#pragma unroll
      for (int t = 0; t < 16; ++t) h[t] = __ldg(th + t);        // all hi-row reads in flight before any is used
#pragma unroll
      for (int t = 0; t < 16; ++t) {
        const float4 l = tl[t];
        const uint64_t ch = ts_pack(h[t].x, h[t].y), sh = ts_pack(h[t].z, h[t].w), cl = ts_pack(l.x, l.y), sl = ts_pack(l.z, l.w);
        cs2[t] = ts_sub(ts_mul(ch, cl), ts_mul(sh, sl));
        sn2[t] = ts_fma(sh, cl, ts_mul(ch, sl));
      }
    };
    auto row_pos = [&](const int4& e) -> int {
      if (cached(e)) return e.x < 0 ? v.joint_pos()[(size_t)~e.x * TILE + row] : kpos[(size_t)e.x * TILE + row];
      if (e.w >= 0 && (e.y & TREE_NODES) && row < (e.y >> 16)) return a.positions[a.info[e.w].x + row];
      return 0;
    };
    TsUnit u = unit(w0);
    if (w0 < total) rope_setup(row_pos(u.e));
    for (int w = w0; w < total && ok; ++w) {
      const TsUnit nxt = unit(w + 1);
      [[maybe_unused]] bool has_row = true;
      if constexpr (DBG) has_row = cached(u.e) ? cache_slot(u.e, row) >= 0 : (u.e.y & TREE_NODES) && row < (u.e.y >> 16);
      const int passes = (u.cls + TS_A_SLOTS - 1) / TS_A_SLOTS;
      const int pos_next = row_pos(nxt.e);                                        // fetched now, used after the tile's slabs
      for (int ps = 0; ps < passes && ok; ++ps) {
        for (int sli = 0; sli < nh; ++sli) {
          if (!(ok = __all_sync(0xffffffffu, mbar_wait(slab_full + 8 * sbuf, sph, abort_flag)))) break;
          fence_after_sync();
          const uint32_t sl_addr = lane_addr + TS_COL_SLAB + sbuf * 128 + hf * 32;
          uint32_t va[16], vb[16];
          tmem_ld8(sl_addr, va);
          tmem_ld8(sl_addr + 64, va + 8);
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            uint32_t* cur = (c & 1) ? vb : va;
            uint32_t* nx = (c & 1) ? va : vb;
            tmem_ld_wait();
            if (c < 3) {
              tmem_ld8(sl_addr + 8 * (c + 1), nx);
              tmem_ld8(sl_addr + 64 + 8 * (c + 1), nx + 8);
            }
            uint32_t oh[8], ol[8];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const int t = 4 * c + k;
              const uint64_t L = ts_pack_bits(cur[2 * k], cur[2 * k + 1]), H = ts_pack_bits(cur[8 + 2 * k], cur[8 + 2 * k + 1]);
              const uint64_t x = ts_sub(ts_mul(L, cs2[t]), ts_mul(H, sn2[t]));           // lo cos - hi sin
              const uint64_t y = ts_fma(L, sn2[t], ts_mul(H, cs2[t]));                   // hi cos + lo sin
              split_pair_16<false>(x, oh[k], ol[k]);
              split_pair_16<false>(y, oh[4 + k], ol[4 + k]);
            }
            if constexpr (DBG) {                                   // a rotated key beyond the f16 range was clamped
              bool sat = false;
#pragma unroll
              for (int k = 0; k < 8; ++k) sat |= (oh[k] & 0x7fffu) == 0x7bffu || ((oh[k] >> 16) & 0x7fffu) == 0x7bffu;
              if (sat && has_row) set_status(v, TWKV_ERR_DEVICE_CHECK);
            }
            tmem_st8(sl_addr + 8 * c, oh);                                    // high parts: columns 0 .. 63 of the slab
            tmem_st8(sl_addr + 64 + 8 * c, ol);                               // low parts: columns 64 .. 127
          }
          tmem_st_wait();
          fence_before_sync();
          __syncwarp();
          if (lane == 0) mbar_arrive_cluster(kr_full_even + 8 * sbuf);
          if (++sbuf == TS_SLABS) { sbuf = 0; sph ^= 1u; }
        }
      }
      if (!ok) break;
      if (nxt.e.w >= 0 && (nxt.e.x != u.e.x || nxt.e.y != u.e.y)) rope_setup(pos_next);      // a further part of the same tile: the factors stay
      u = nxt;
    }
    tmem_ld_wait();                                                          // nothing of this thread is in flight when TMEM is freed
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(TS_REGS_OUT));
    // ------------------------------------------------------------- scores out
    // One warp per TMEM lane quarter.  32 columns at a time: a thread reads its token row, the warp turns the block in shared memory (rows
    // of 128 bytes, 16-byte pieces swizzled), then eight lanes hold a row and store it as whole lines; a lane meets four columns of eight
    // rows on the way, whose maxima the warp joins.  The maxima in memory are read ahead, and only a larger one is sent there.
    const int quarter = warp & 3, row = quarter * 32 + lane, sub_row = lane >> 3, piece4 = lane & 7;
    const uint32_t lane_addr = tmem_base + ((uint32_t)(quarter * 32) << 16);
    float4* stage = reinterpret_cast<float4*>(out_stage + quarter * TS_OUT_WARP);
    const float sm_scale = v.sm_scale;
    const int rep_shift = __ffs(v.rep) - 1;
    uint32_t slot = 0, slph = 0;
    bool ok = true;
    auto score_row = [&](const int4& e) -> int {                   // -1: no token
      if (cached(e)) {
        const int k = cache_slot(e, row);
        return k >= 0 ? v.kv_link[k] : -1;
      }
      return e.w >= 0 && (e.y & TREE_NODES) && row < (e.y >> 16) ? e.x * TILE + row : -1;
    };
    TsUnit u = unit(w0);
    int srow = score_row(u.e);
    for (int w = w0; w < total && ok; ++w) {
      const TsUnit nxt = unit(w + 1);
      const int srow_next = score_row(nxt.e);
      const int passes = (u.cls + TS_A_SLOTS - 1) / TS_A_SLOTS, g0 = first_head(w);
      const bool node = (u.e.y & TREE_NODES) != 0, drop = (u.e.y & TREE_FILLER) != 0;
      const int4 info = node ? a.info[u.e.w] : make_int4(0, 0, 0, 0);
      int dst_row[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) dst_row[k] = __shfl_sync(0xffffffffu, srow, 4 * k + sub_row);
      for (int ps = 0; ps < passes && ok; ++ps) {
        const bool add = ps > 0, last = ps == passes - 1;
        for (int sli = 0; sli < nh && ok; ++sli) {
          const int g = head(g0, sli);
          for (int sub = 0; sub < n_sub; ++sub) {
            const int cols = min(TS_QCOLS, a.Rs - sub * TS_QCOLS);             // columns to store, a multiple of four (none: only operand padding)
            const int c_base = g * a.Rs + sub * TS_QCOLS;
            unsigned* const top = a.seqmax + (size_t)(u.e.w) * a.C + c_base;
            if (!(ok = __all_sync(0xffffffffu, mbar_wait(s_full + 8 * slot, slph, abort_flag)))) break;
            fence_after_sync();
            const uint32_t src = lane_addr + TS_COL_S + TS_QCOLS * slot;
            const int chunks = cols > 32 ? 2 : 1;
            for (int ch = 0; ch < chunks; ++ch) {
              float x[32];
              tmem_ld32(src + 32 * ch, x);
              const unsigned seen = !drop && last && 32 * ch + lane < cols ? *(volatile unsigned*)(top + 32 * ch + lane) : 0xffffffffu;
              tmem_ld_wait();
              if (ch == chunks - 1) {
                fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(s_empty_even + 8 * slot);
              }
              if (drop) continue;
#pragma unroll
              for (int c = 0; c < 32; ++c) x[c] *= sm_scale;
              if (node) {                                          // a node is seen by the queries whose masks hold its bit
#pragma unroll
                for (int c = 0; c < 32; ++c) {
                  const int t = (sub * TS_QCOLS + 32 * ch + c) >> rep_shift;
                  const unsigned long long m = t < info.y ? a.masks[info.x + t] : 0ull;
                  if (!((m >> (row & 63)) & 1ull)) x[c] = -INFINITY;
                }
              }
#pragma unroll
              for (int c = 0; c < 8; ++c) stage[lane * 8 + (c ^ (lane & 7))] = make_float4(x[4 * c], x[4 * c + 1], x[4 * c + 2], x[4 * c + 3]);
              __syncwarp();
              const bool mine = 32 * ch + 4 * piece4 < cols;
              float* const dst = a.scores + c_base + 32 * ch + 4 * piece4;
              float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
              for (int k = 0; k < 8; ++k) {
                const int r = 4 * k + sub_row;
                float4 y = stage[r * 8 + (piece4 ^ (r & 7))];
                if (mine && dst_row[k] >= 0) {
                  float4* p = reinterpret_cast<float4*>(dst + (size_t)dst_row[k] * a.C);
                  if (add) {                                       // (this thread stored the first pass's part)
                    const float4 o = *p;
                    y.x += o.x; y.y += o.y; y.z += o.z; y.w += o.w;
                  }
                  *p = y;
                  mx[0] = fmaxf(mx[0], y.x); mx[1] = fmaxf(mx[1], y.y); mx[2] = fmaxf(mx[2], y.z); mx[3] = fmaxf(mx[3], y.w);
                }
              }
              __syncwarp();                                        // the block has been read
              if (!last) continue;
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                mx[e] = fmaxf(mx[e], __shfl_xor_sync(0xffffffffu, mx[e], 8));
                mx[e] = fmaxf(mx[e], __shfl_xor_sync(0xffffffffu, mx[e], 16));
              }
              // lane = column: the maximum of column 4 (lane / 4) + lane % 4 sits in the lanes of piece lane / 4
              float m = -INFINITY;
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const float t = __shfl_sync(0xffffffffu, mx[e], lane >> 2);
                if ((lane & 3) == e) m = t;
              }
              const unsigned enc = enc_ordered(m);
              if (enc > seen) atomicMax(top + 32 * ch + lane, enc);
            }
            if (++slot == TS_S_SLOTS) { slot = 0; slph ^= 1u; }
          }
        }
      }
      srow = srow_next;
      u = nxt;
    }
    tmem_ld_wait();                                                          // nothing of this thread is in flight when TMEM is freed
  }

  fence_before_sync();
  __syncthreads();
  cluster_sync_all();                                           // the partner is done with this CTA's memory and barriers as well
  fence_after_sync();
  if (warp == 1) tmem_dealloc_pair(tmem_base, 512);
  if (tid == 0 && *abort_flag) set_status(v, misaligned ? TWKV_ERR_DEVICE_CHECK : TWKV_ERR_TIMEOUT);
}

// CTA pairs that can be resident at once on the current device (0: the kernel cannot run).
static int tree_query_pairs(int sm_count) {
  auto kernel = tree_score_kernel<false, false>;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)TS_SMEM) != cudaSuccess) { cudaGetLastError(); return 0; }
  cudaLaunchConfig_t cfg = {};
  cfg.blockDim = dim3(TS_THREADS);
  cfg.dynamicSmemBytes = TS_SMEM;
  cfg.gridDim = dim3(sm_count & ~1);
  cudaLaunchAttribute pair_attr;
  pair_attr.id = cudaLaunchAttributeClusterDimension;
  pair_attr.val.clusterDim.x = 2; pair_attr.val.clusterDim.y = 1; pair_attr.val.clusterDim.z = 1;
  cfg.attrs = &pair_attr;
  cfg.numAttrs = 1;
  int n = 0;
  if (cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess || n < 1) { cudaGetLastError(); n = 0; }
  return n;
}
int tree_max_pairs(int sm_count) {
  static const int cached = tree_query_pairs(sm_count);         // queried once per process (thread-safe initialisation)
  return cached;
}

int tree_query_box(const TreeCall& a) { return a.Rp / 2 < TS_QCOLS / 2 ? a.Rp / 2 : TS_QCOLS / 2; }

cudaError_t launch_tree_score(const DevView& v, const TreeCall& a, const TreeMaps& maps, int layer, int n_pieces, cudaStream_t st) {
  ProfScope ps(TWKV_K_KSCORE, st);
  auto kernel = v.dtype == TWKV_BF16 ? (v.debug ? tree_score_kernel<true, true> : tree_score_kernel<true, false>)
                                     : (v.debug ? tree_score_kernel<false, true> : tree_score_kernel<false, false>);
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)TS_SMEM);
  if (e != cudaSuccess) return e;
  e = launch_chained(kernel, dim3(2 * n_pieces), dim3(TS_THREADS), dim3(2), TS_SMEM, st, maps.blocks, maps.boxes, maps.nodes, maps.uinvT, maps.q, v, a, layer);
  if (e != cudaSuccess) return e;
  count_launch();
  return cudaGetLastError();
}

}  // namespace twkv
