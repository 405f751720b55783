// Scores of drafted trees on the 5th-generation tensor cores.
//
// Per K tile (128 tokens, c panels) and KV head g, as in a decode pass (kscore_tc.cu):
//   Kbar_g = X^_K U_K^-1[:, g]  (Eq. 3),  Krot_g = RoPE(Kbar_g),  S_g = Krot_g Q_g^T
// with all query rows of the request, nodes x heads of the group, in Q_g.  A tile is rebuilt and rotated once for all of them; that is
// what a pass of single queries per node repeats.  The kernel runs on CTA pairs (M = 256 over two tiles of ONE request, so that
// each CTA holds half of Q_g's rows and every column of the product is wanted).  Query rows go through in blocks of 64 columns
// (N = 16 .. 64): their operand, made by the plan kernel, streams through a ring, a block's scores land in one of two accumulators (four of 32
// columns where that is all there is).
//
// Tensor memory (512 columns): slabs of rebuilt keys 3 x 128 | score accumulators 2 x 64.
// Warp roles (512 threads, one persistent CTA per SM; registers re-divided by warpgroup):
//   warp 0      TMA producer of U_K^-1 panels
//   warp 1      issuer of the reconstruction products (even CTA; owns the TMEM allocation)
//   warp 2      TMA producer of X^_K panels and of the query blocks
//   warp 3      issuer of the score products (even CTA)
//   warps 4-11  rotation and high / low split (thread = one token row x half of the RoPE frequencies)
//   warps 12-15 scores out: masked (nodes), stored in the order of the V tiles (thread = one token row)
// Measured: 64 sequences of 8192 tokens with 8 nodes (32 query heads, fp16) 530 us, 410 in a call by itself: the power cap, as in a decode pass.  Tensor pipe
// 46 %, issue slots 26 % and memory 2.3 TB/s in a short call: a key's way through rebuilding, rotation, product and store bounds it there.
// Scores are stored without their scale, which the value kernel's exponents carry (a negative scale is in the queries).
// A class wider than eight panels runs as two passes over its panels (unless there are many query rows, see panels()), the second adding to the scores
// the first one stored (one addition per score, in memory: its order cannot vary).
// All waits are bounded (tc_util.cuh); a wait that runs out ends the kernel with TWKV_ERR_TIMEOUT.
#include "twkv_dev.h"
#include "tc_util.cuh"
#include "tree.h"

namespace twkv {
using namespace tc;

constexpr int TS_THREADS = 512;
constexpr int TS_REGS_LIGHT = 56, TS_REGS_EPI = 184, TS_REGS_OUT = 88;      // 128 x 56 + 256 x 184 + 128 x 88 = 65536
constexpr int TS_A_SLOTS = 8, TS_B_STAGES = 4, TS_SLABS = 3;
constexpr int TS_Q_STAGES = 6;                                  // stages of the query ring where a block has at most 32 rows, half as many where it has 64
constexpr int TS_STREAM_ROWS = 64;                              // query rows beyond which a class of more than eight panels is rebuilt in one pass
constexpr int TS_S_SLOTS = 4;                                   // score accumulators of 32 columns, or half as many of 64
constexpr uint32_t TS_PANEL = 16384, TS_B_PART = 8192, TS_B_STAGE = 2 * TS_B_PART;
constexpr int TS_QCOLS = 64;                                    // query rows of a block, half of them in each CTA
constexpr uint32_t TS_Q_BYTES = 3 * TS_QCOLS / 2 * 256;          // the ring: three blocks of 64 rows, this CTA's half of each
constexpr uint32_t TS_COL_SLAB = 0, TS_COL_S = 128 * TS_SLABS;
constexpr int TS_ROPE_STRIDE = 33;                              // float4 per row of the small RoPE table (32 + 1 against bank conflicts)
constexpr uint32_t TS_ROPE_BYTES = ROPE_LO * TS_ROPE_STRIDE * 16;
constexpr int TS_N_BARS = 2 * TS_A_SLOTS + 2 * TS_B_STAGES + 2 * TS_Q_STAGES + 3 * TS_SLABS + 2 * TS_S_SLOTS;
constexpr uint32_t TS_SMEM = TS_A_SLOTS * TS_PANEL + TS_B_STAGES * TS_B_STAGE + TS_Q_BYTES + TS_ROPE_BYTES + 8 * TS_N_BARS + 16;
static_assert(TS_SMEM > CHAIN_TMEM_SMEM && TS_SMEM <= 232448, "no other CTA with tensor memory beside this one");
static_assert(TS_COL_S + TS_QCOLS / 2 * TS_S_SLOTS <= 512, "tensor memory");

__device__ __forceinline__ uint64_t ts_pack(float a, float b) { uint64_t r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ uint64_t ts_pack_bits(uint32_t a, uint32_t b) { uint64_t r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "r"(a), "r"(b)); return r; }
__device__ __forceinline__ uint64_t ts_mul(uint64_t a, uint64_t b) { uint64_t r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ uint64_t ts_sub(uint64_t a, uint64_t b) { uint64_t r; asm("sub.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ uint64_t ts_fma(uint64_t a, uint64_t b, uint64_t c) { uint64_t r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }

// Whether the phase has completed, without waiting for it.
__device__ __forceinline__ bool mbar_test(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok != 0;
}
// Looks at both rings without finding room after which the producer gives up: a look takes a few dozen cycles, so a second or more.
constexpr uint32_t TS_IDLE_LIMIT = 1u << 26;

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
  float4* sRope = reinterpret_cast<float4*>(smem_raw + TS_A_SLOTS * TS_PANEL + TS_B_STAGES * TS_B_STAGE + TS_Q_BYTES);
  unsigned char* tail = reinterpret_cast<unsigned char*>(sRope) + TS_ROPE_BYTES;
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
  const uint32_t s_cols = a.Rp <= TS_QCOLS / 2 ? TS_QCOLS / 2 : TS_QCOLS, s_slots = a.Rp <= TS_QCOLS / 2 ? TS_S_SLOTS : TS_S_SLOTS / 2;
  const uint32_t q_stages = a.Rp <= TS_QCOLS / 2 ? TS_Q_STAGES : TS_Q_STAGES / 2, q_stage = TS_Q_BYTES / q_stages, q_panel = q_stage / 2;
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
  // panels of a pass: eight, which stay in their ring slots for all KV heads of the unit; all, brought once per KV head, where a class is wider and
  // there are so many query rows that rotating, multiplying and storing twice costs more
  auto panels = [&](int cls) -> int { return a.R > TS_STREAM_ROWS && cls > TS_A_SLOTS ? cls : TS_A_SLOTS; };
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
      // ----------------------------------------------------------- TMA producer: X^_K panels and query blocks
      // Two queues of copies with a ring each, in the order of their use; one thread looks at the rings in turn and issues what has
      // room, so that neither waits for the other.  (A producer of the blocks inside the issuer of their products cost that thread a
      // quarter of its time, one inside the warps that store the scores their registers.)
      if (elect_one()) {
        tma_prefetch_desc(&map_blocks);
        tma_prefetch_desc(&map_boxes);
        tma_prefetch_desc(&map_nodes);
        tma_prefetch_desc(&map_q);
        // panels: unit w, panel j, times the unit's panels have been brought, panels so far ak (slot = ak % 8); blocks: unit lw, first panel of the
        // pass lp, KV head lsl, block lsub
        int w = w0, j = 0, again = 0, lw = w0, lp = 0, lsl = 0, lsub = 0;
        uint32_t ak = 0, lst = 0, lph = 0, idle = 0;
        TsUnit u = unit(w0), lu = u;
        while (w < total || lw < total) {
          bool moved = false;
          if (w < total && mbar_test(a_empty + 8 * (ak % TS_A_SLOTS), ((ak / TS_A_SLOTS) & 1u) ^ 1u)) {
            const uint32_t slot = ak % TS_A_SLOTS, dst = sA + slot * TS_PANEL;
            const int own = u.e.y & TREE_CLASS;
            if (crank == 0) mbar_expect_tx(a_full + 8 * slot, 2 * TS_PANEL);            // this CTA's copy and the partner's
            if (u.e.x < 0) {
              const unsigned* box = v.joint_boxes() + (size_t)~u.e.x * (TILE / JOINT_ROWS);
#pragma unroll
              for (int b = 0; b < TILE / JOINT_ROWS; ++b) {     // a box of a narrower class lies behind the last block from its class on and reads zeros there
                const unsigned x = box[b];
                tma_load_2d_pair(dst + b * (JOINT_ROWS * PANEL * 2), &map_boxes, a_full_even + 8 * slot, 0,
                                 j < (int)(x & 31u) ? (int)(x >> 5) * JOINT_ROWS + j * TILE : v.n_blocks * TILE);
              }
            } else if ((u.e.y & TREE_NODES) && j < own) {
              tma_load_2d_pair(dst, &map_nodes, a_full_even + 8 * slot, 0, u.e.z + j * TREE_PANEL_ROWS);       // rows past the nodes': other panels, dropped
            } else {
              tma_load_2d_pair(dst, &map_blocks, a_full_even + 8 * slot, 0, j < own ? (u.e.z + j) * TILE : v.n_blocks * TILE);
            }
            ++ak;
            if (++j == u.cls) {
              j = 0;
              if (panels(u.cls) > TS_A_SLOTS && ++again < nh) continue;         // the panels of a streamed unit's next KV head
              again = 0;
              u = unit(++w);
            }
            moved = true;
          }
          if (lw < total && mbar_test(q_empty + 8 * lst, lph ^ 1u)) {
            const int half = min(TS_QCOLS, a.Rp - lsub * TS_QCOLS) / 2;
            const int y = (lu.e.w * v.Hkv + head(first_head(lw), lsl)) * a.Rp + lsub * TS_QCOLS + (int)crank * half;
            if (crank == 0) mbar_expect_tx(q_full + 8 * lst, 2 * 2 * (uint32_t)a.q_box * 128u);
            tma_load_2d_pair(sQ + lst * q_stage, &map_q, q_full_even + 8 * lst, 0, y);
            tma_load_2d_pair(sQ + lst * q_stage + q_panel, &map_q, q_full_even + 8 * lst, PANEL, y);
            if (++lst == q_stages) { lst = 0; lph ^= 1u; }
            if (++lsub == n_sub) {
              lsub = 0;
              if (++lsl == nh) {
                lsl = 0;
                lp += panels(lu.cls);
                if (lp >= lu.cls) { lp = 0; lu = unit(++lw); }
              }
            }
            moved = true;
          }
          idle = moved ? 0u : idle + 1u;
          if (!moved) __nanosleep(100);
          if ((idle & 63u) == 63u) {
            if (*abort_flag) break;
            if (idle > TS_IDLE_LIMIT) { *abort_flag = 1; break; }
          }
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
          const int span = panels(u.cls);
          for (int p0 = 0; p0 < u.cls && ok; p0 += span) {
            const int np = min(span, u.cls - p0);
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
          const int span = panels(u.cls);
          const bool stream = span > TS_A_SLOTS;
          for (int p0 = 0; p0 < u.cls && ok; p0 += span) {
            const int np = min(span, u.cls - p0);
            for (int sl = 0; sl < nh && ok; ++sl) {
              // the buffer is free once the score products over its previous contents have retired
              if (!(ok = mbar_wait_thin(slab_empty + 8 * sbuf, sph ^ 1u, abort_flag))) break;
              fence_after_sync();
              const uint32_t d = tmem_base + TS_COL_SLAB + sbuf * 128;
              const bool first = stream || sl == 0, last = stream || sl == nh - 1;
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
              if (last) ak += np;
            }
          }
          u = nxt;
        }
      }
      __syncwarp();
    } else {
      // ----------------------------------------------------------- issuer of the score products
      if (crank == 0 && elect_one()) {
        const uint32_t q_lo0 = kmajor_sw128_desc_lo(sQ);
        uint32_t sbuf = 0, sph = 0, slot = 0, slph = 0, qst = 0, qph = 0;
        bool ok = true;
        TsUnit u = unit(w0);
        for (int w = w0; w < total && ok; ++w) {
          const TsUnit nxt = unit(w + 1);
          for (int p0 = 0; p0 < u.cls && ok; p0 += panels(u.cls)) {
            for (int sl = 0; sl < nh && ok; ++sl) {
              if (!(ok = mbar_wait_thin(kr_full + 8 * sbuf, sph, abort_flag))) break;
              const uint32_t kr = tmem_base + TS_COL_SLAB + sbuf * 128;
              for (int sub = 0; sub < n_sub; ++sub) {
                if (!(ok = mbar_wait_thin(s_empty + 8 * slot, slph ^ 1u, abort_flag))) break;
                if (!(ok = mbar_wait_thin(q_full + 8 * qst, qph, abort_flag))) break;
                fence_after_sync();
                const uint32_t idesc_s = idesc_f16(0, 256, min(TS_QCOLS, a.Rp - sub * TS_QCOLS));
                const uint32_t sd = tmem_base + TS_COL_S + s_cols * slot, ql = q_lo0 + qst * (q_stage >> 4);
                // high and low f16 parts of the rotated keys into the same accumulator, the low one first
                mma_f16_ts_k128_cg<2>(sd, kr + 64, ql, q_panel >> 4, idesc_s, 0u);
                mma_f16_ts_k128_cg<2>(sd, kr, ql, q_panel >> 4, idesc_s, 1u);
                mma_commit_pair_both(q_empty + 8 * qst);
                if (sub == n_sub - 1) mma_commit_pair(slab_empty + 8 * sbuf);
                mma_commit_pair_both(s_full + 8 * slot);
                if (++slot == s_slots) { slot = 0; slph ^= 1u; }
                if (++qst == q_stages) { qst = 0; qph ^= 1u; }
              }
              if (++sbuf == TS_SLABS) { sbuf = 0; sph ^= 1u; }
            }
          }
          u = nxt;
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
    auto rope_setup = [&](int2 at) {                               // position, class of the row
      const int pos = at.x, chain = 4 * min(at.y, panels(at.y));   // instructions that a key of the row was summed in
      const uint64_t up = ts_pack(1.f + TREE_CUT * (float)chain, 1.f + TREE_CUT * (float)chain);
      const float4* __restrict__ th = rope_hi + (size_t)((pos >> 4) & (ROPE_HI - 1)) * 32 + hf * 16;
      const float4* tl = sRope + (pos & 15) * TS_ROPE_STRIDE + hf * 16;
      float4 h[16];
#pragma unroll
      for (int t = 0; t < 16; ++t) h[t] = __ldg(th + t);        // all hi-row reads in flight before any is used
#pragma unroll
      for (int t = 0; t < 16; ++t) {
        const float4 l = tl[t];
        const uint64_t ch = ts_pack(h[t].x, h[t].y), sh = ts_pack(h[t].z, h[t].w), cl = ts_pack(l.x, l.y), sl = ts_pack(l.z, l.w);
        cs2[t] = ts_mul(ts_sub(ts_mul(ch, cl), ts_mul(sh, sl)), up);
        sn2[t] = ts_mul(ts_fma(sh, cl, ts_mul(ch, sl)), up);
      }
    };
    auto row_at = [&](const int4& e) -> int2 {
      const int cls = e.y & TREE_CLASS;
      if (cached(e) && e.x < 0) {
        const int k = v.joint_rows()[(size_t)~e.x * TILE + row];
        return make_int2(v.joint_pos()[(size_t)~e.x * TILE + row], k >= 0 ? v.desc(layer, 0)[k / TILE].y : cls);
      }
      if (cached(e)) return make_int2(kpos[(size_t)e.x * TILE + row], cls);
      if (e.w >= 0 && (e.y & TREE_NODES) && row < (e.y >> 16)) return make_int2(a.positions[a.info[e.w].x + row], cls);
      return make_int2(0, cls);
    };
    TsUnit u = unit(w0);
    if (w0 < total) rope_setup(row_at(u.e));
    for (int w = w0; w < total && ok; ++w) {
      const TsUnit nxt = unit(w + 1);
      [[maybe_unused]] bool has_row = true;
      if constexpr (DBG) has_row = cached(u.e) ? cache_slot(u.e, row) >= 0 : (u.e.y & TREE_NODES) && row < (u.e.y >> 16);
      const int passes = u.cls > panels(u.cls) ? 2 : 1;
      const int2 at_next = row_at(nxt.e);                                         // fetched now, used after the tile's slabs
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
      if (nxt.e.w >= 0 && (nxt.e.x != u.e.x || nxt.e.y != u.e.y)) rope_setup(at_next);      // a further part of the same tile: the factors stay
      u = nxt;
    }
    tmem_ld_wait();                                                          // nothing of this thread is in flight when TMEM is freed
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(TS_REGS_OUT));
    // ------------------------------------------------------------- scores out
    // One warp per TMEM lane quarter, thread = token row: 32 columns at a time go straight to the token's score row, in pieces of 32 bytes.  A
    // single warp issues an instruction every five cycles or so, and a slab leaves it about 2000: this loop is kept short, the
    // maxima are the value kernel's.  (Turned in shared memory, so that lanes share a row, with maxima by column, a block of 32 columns took
    // 1475 cycles; sent off as TMA boxes 1900.)
    const int quarter = warp & 3, row = quarter * 32 + lane;
    const uint32_t lane_addr = tmem_base + ((uint32_t)(quarter * 32) << 16) + TS_COL_S;
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
      const int passes = u.cls > panels(u.cls) ? 2 : 1, g0 = first_head(w);
      const bool live = srow >= 0;                                 // (a filler's rows are not)
      float* const dst_row = a.scores + (size_t)(live ? srow : 0) * a.C;
      const bool node = (u.e.y & TREE_NODES) != 0;
      const unsigned long long seers = node ? a.seers[(size_t)u.e.w * TWKV_TREE_MAX_NODES + (row & (TWKV_TREE_MAX_NODES - 1))] : ~0ull;
      const int srow_next = score_row(nxt.e);
      for (int ps = 0; ps < passes && ok; ++ps) {
        for (int sli = 0; sli < nh && ok; ++sli) {
          const int g = head(g0, sli);
          for (int sub = 0; sub < n_sub; ++sub) {
            const int cols = min(TS_QCOLS, a.Rs - sub * TS_QCOLS);
            float* const dst = dst_row + g * a.Rs + sub * TS_QCOLS;
            if (!(ok = __all_sync(0xffffffffu, mbar_wait(s_full + 8 * slot, slph, abort_flag)))) break;
            fence_after_sync();
            const uint32_t src = lane_addr + s_cols * slot;
#pragma unroll
            for (int ch = 0; ch < 2; ++ch) {
              if (32 * ch >= cols) break;
              uint32_t x[32];
              tmem_ld32(src + 32 * ch, x);
              tmem_ld_wait();
              if (32 * ch + 32 >= cols) {                          // the accumulator has been read
                fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(s_empty_even + 8 * slot);
              }
              if (node) {                                          // a node is seen by the queries whose masks hold its bit
                const unsigned bits = (unsigned)(seers >> ((sub * TS_QCOLS + 32 * ch) >> rep_shift));       // (32 columns are at most 32 nodes)
#pragma unroll
                for (int c = 0; c < 32; ++c)
                  if (!((bits >> (c >> rep_shift)) & 1u)) x[c] = 0xff800000u;
              }
              if (live && ps > 0) {                                // onto what this thread stored of the first pass
#pragma unroll
                for (int c = 0; c < 8; ++c)
                  if (32 * ch + 4 * c < cols)
                    asm volatile("red.global.add.v4.f32 [%0], {%1, %2, %3, %4};" ::"l"(__cvta_generic_to_global(dst + 32 * ch + 4 * c)), "f"(__uint_as_float(x[4 * c])),
                                 "f"(__uint_as_float(x[4 * c + 1])), "f"(__uint_as_float(x[4 * c + 2])), "f"(__uint_as_float(x[4 * c + 3])) : "memory");
              } else if (live) {
                if (a.Rs >= 8) {
#pragma unroll
                  for (int c = 0; c < 4; ++c)
                    if (32 * ch + 8 * c < cols)
                      asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                                   ::"l"(__cvta_generic_to_global(dst + 32 * ch + 8 * c)), "r"(x[8 * c]), "r"(x[8 * c + 1]), "r"(x[8 * c + 2]), "r"(x[8 * c + 3]),
                                     "r"(x[8 * c + 4]), "r"(x[8 * c + 5]), "r"(x[8 * c + 6]), "r"(x[8 * c + 7]) : "memory");
                } else if (ch == 0) {
                  *reinterpret_cast<uint4*>(dst) = make_uint4(x[0], x[1], x[2], x[3]);
                }
              }
            }
            if (++slot == s_slots) { slot = 0; slph ^= 1u; }
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
