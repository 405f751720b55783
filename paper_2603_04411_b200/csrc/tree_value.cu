// Weighted values of drafted trees on the 5th-generation tensor cores.
//
// As in a decode pass (vacc_tc.cu) the weighted sum is taken in spectral space, for 128 query rows c = (KV head, node, head of the group):
//   acc[c][j] = sum over the split's tokens t of p[t][c] X^_V[t][j],   p = exp(s - top[c]),   l[c] = sum of p[t][c]
// The weights are the A operand, from tensor memory (M = 128 query rows, K = 16 tokens per instruction), and the panels of a V tile, as TMA lands
// them, the MN-major B operand (N = 128: two panels): a panel is read from shared memory once per 128 rows and part of the weights, which come as
// two parts of the cache type, or three where a bf16 cache has fp32 outputs.  (One part, with room for the weights of two tiles, gains 5 % at the
// most: the weights' instructions and memory bound the kernel.  With the panels as A and 64 columns of weights as B, both from shared memory, an
// instruction of half the work took 85 cycles for its operands instead of 32: 12200 cycles per tile of sixteen panels and 64 columns.)
// Tensor memory holds the weights of one tile (64 columns per part) and three accumulators of 128 columns: six panels (with three parts two: four).  A
// CTA therefore takes a range of six panels (blockIdx.z); the higher ranges, which only wide tiles reach, form those tiles' weights again.
// A tile's scores come by TMA while the tile before is worked on (read from memory by the lanes themselves, whose registers hold one tile, their
// latency bound the kernel: 5600 cycles per narrow tile).  What a row's weights are relative to, top[c], is its largest score so far (fp16: 2^-7 of it,
// so that what is 2^31 below the maximum is still more than zero), moved only when that has grown by more than 2^8 (f16 holds 2^15): the accumulators
// are rescaled seldom, by the warps that own their lanes.  The merge brings the splits' parts together.
// A tile of four panels takes 2.4 to 2.7 us (16 sequences of 32768 tokens, 128 CTAs), of which the products are 1.1: 8900 warp instructions form its
// 16384 weights, 48 % of the issue slots of that time.
// Tiles that are at most half full, and the nodes' tile, are read by the boxes of sixteen rows that hold tokens.
//
// Warp roles (640 threads, one CTA per SM): 0 TMA producer of V panels, 1 MMA issuer (owns the TMEM allocation), 2 TMA producer of scores, 4-19 weights
// (quarter = warp % 4 of the rows, part (warp - 4) / 4 of the tile's tokens), then the read-out.
// All waits are bounded (tc_util.cuh); a wait that runs out ends the kernel with TWKV_ERR_TIMEOUT.
#include "twkv_dev.h"
#include "tc_util.cuh"
#include "tree.h"

namespace twkv {
using namespace tc;

constexpr int TV_THREADS = 640;
constexpr int TV_REGS_LIGHT = 64, TV_REGS_WEIGHTS = 104;       // 128 x 64 + 512 x 104 = 61440 = 640 x 96
constexpr int TV_META = 256;                                   // tiles whose descriptors are staged in shared memory at a time
constexpr int TV_STAGES = 4;
constexpr uint32_t TV_PANEL = 16384, TV_STAGE = 2 * TV_PANEL;
constexpr uint32_t TV_SCORES = TILE * TILE * 4;                 // a tile's scores with 128 query rows
constexpr uint32_t TV_SMEM = TV_STAGES * TV_STAGE + TV_SCORES + TV_META * 16 + (2 + 2) * 4 * TILE * 4 + 256;
static_assert(TV_SMEM > CHAIN_TMEM_SMEM && TV_SMEM <= 232448, "no other CTA with tensor memory beside this one");
static_assert(2 * TREE_PANEL_ROWS <= TILE, "the nodes' tile always comes in boxes");

constexpr float TV_SMALL = 24.f;                               // bits of an fp32 sum
static_assert(2 * (TREE_DRAIN_16 + TILE / JOINT_ROWS) < 65536, "lossy instructions of an accumulator, in sixteen bits");
constexpr float TV_LOG2E = 1.44269504088896340736f;
__device__ __forceinline__ uint64_t tv_pack(float a, float b) { uint64_t r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ void tv_unpack(uint64_t v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t tv_fma2(uint64_t a, uint64_t b, uint64_t c) { uint64_t r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }
__device__ __forceinline__ uint64_t tv_add2(uint64_t a, uint64_t b) { uint64_t r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ float tv_ex2(float x) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }

// PARTS = 2: three accumulators of two panels, then the weights (2 x 64 columns); 3: two accumulators and 3 x 64 columns.
__host__ __device__ constexpr int tv_range(int parts) { return parts == 3 ? 4 : 6; }
int tree_value_range(int parts) { return tv_range(parts); }
static_assert((TWKV_MAX_CLASSES + tv_range(3) - 1) / tv_range(3) <= TREE_MAX_RANGES, "a reference per range");
static_assert(tv_range(2) * 64 + 2 * 64 <= 512 && tv_range(3) * 64 + 3 * 64 <= 512, "tensor memory");

__device__ __forceinline__ void tv_ld8(const float* p, float* x) {
  asm volatile("ld.global.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]), "=f"(x[4]), "=f"(x[5]), "=f"(x[6]), "=f"(x[7]) : "l"(__cvta_generic_to_global(p)) : "memory");
}
__device__ __forceinline__ void tv_st8(float* p, const float* x) {
  asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               ::"l"(__cvta_generic_to_global(p)), "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7]) : "memory");
}

template <bool BF16, int PARTS>
__global__ void __launch_bounds__(TV_THREADS, 1)
tree_value_kernel(const __grid_constant__ CUtensorMap map_blocks, const __grid_constant__ CUtensorMap map_boxes, const __grid_constant__ CUtensorMap map_nodes,
                  const __grid_constant__ CUtensorMap map_scores, const __grid_constant__ CUtensorMap map_score_boxes, DevView v, TreeCall a) {
  constexpr int RANGE = tv_range(PARTS), COLS = RANGE * PANEL;
  constexpr uint32_t COL_P = COLS;
  constexpr float HEAD = BF16 ? 0.f : 7.f;                       // powers of two that the largest weight has when top is set
  chain_start();
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int req = blockIdx.x / a.n_splits, split = blockIdx.x - req * a.n_splits, c0 = blockIdx.y * TILE, range = blockIdx.z, panel0 = range * RANGE;
  // shared memory: ring | scores [128 tokens][columns of a box] | descriptors | maxima [2][4 parts][128 rows] | lossy instructions [2][4][128] | barriers
  const uint32_t sRing = smem_addr(smem_raw);
  const bool misaligned = (sRing & 1023u) != 0;                 // operand tiles need 1024-byte alignment for the swizzle
  const float* s_scores = reinterpret_cast<const float*>(smem_raw + TV_STAGES * TV_STAGE);
  const uint32_t sScores = sRing + TV_STAGES * TV_STAGE;
  int4* s_meta = reinterpret_cast<int4*>(smem_raw + TV_STAGES * TV_STAGE + TV_SCORES);
  float* s_max = reinterpret_cast<float*>(s_meta + TV_META);
  uint32_t* s_lossy = reinterpret_cast<uint32_t*>(s_max + 2 * 4 * TILE);
  unsigned char* tail = reinterpret_cast<unsigned char*>(s_lossy + 2 * 4 * TILE);
  const uint32_t bars = smem_addr(tail);
  const uint32_t full = bars, empty = full + 8 * TV_STAGES, p_full = empty + 8 * TV_STAGES, p_done = p_full + 8, sc_full = p_done + 8, sc_empty = sc_full + 8;
  uint32_t* s_tmem_base = reinterpret_cast<uint32_t*>(tail + 8 * (2 * TV_STAGES + 4));
  volatile int* abort_flag = reinterpret_cast<int*>(s_tmem_base + 1);
  volatile int* s_count = abort_flag + 1;                       // [2] tiles of the chunk that reach the range, widest class of the split
  if (tid == 0) {
    for (int i = 0; i < TV_STAGES; ++i) { mbar_init(full + 8 * i, 1); mbar_init(empty + 8 * i, 1); }
    mbar_init(p_full, 16);
    mbar_init(p_done, 1);
    mbar_init(sc_full, 1);
    mbar_init(sc_empty, 16);
    *abort_flag = misaligned ? 1 : 0;
    s_count[1] = 0;
    mbar_init_fence();
  }
  if (warp == 1) tmem_alloc(smem_addr(s_tmem_base), 512);
  fence_before_sync();
  __syncthreads();
  fence_after_sync();
  const uint32_t tmem_base = *s_tmem_base;

  chain_wait();
  const int4 info = a.info[req];
  const int* cut = a.vcut + (size_t)req * (a.n_splits + 1) + split;
  const int t_first = cut[0], n_mine = misaligned ? 0 : cut[1] - t_first;
  const int4* meta = a.vmeta + (size_t)req * (v.TPS + 1) + t_first;

  // k counts the tiles that reach the range; the roles take the split's descriptors a chunk at a time, together
  uint32_t k = 0, touched = 0;                                  // touched: accumulators that hold a value (issuer: has written; weight warps: will have)
  bool ok = true;
  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(TV_REGS_LIGHT));
    uint32_t st = 0, st_ph = 0, n_loaded = 0;                   // ring stage and its phase; stages filled so far
    int since = 0;                                              // boxes of tokens in the accumulators
    for (int k0 = 0; k0 < n_mine; k0 += TV_META) {
      if (warp == 0) {
        // the chunk's tiles that reach the range, in order
        int n = 0, cls = 0;
        int4 m[TV_META / 32];
#pragma unroll
        for (int i = 0; i < TV_META / 32; ++i) m[i] = k0 + 32 * i + lane < n_mine ? meta[k0 + 32 * i + lane] : make_int4(0, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < TV_META / 32; ++i) {
          const unsigned mine = __ballot_sync(0xffffffffu, m[i].y > panel0);
          if (m[i].y > panel0) s_meta[n + __popc(mine & ((1u << lane) - 1u))] = m[i];
          n += __popc(mine);
          cls = max(cls, m[i].y);
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) cls = max(cls, __shfl_xor_sync(0xffffffffu, cls, o));
        if (lane == 0) { s_count[0] = n; s_count[1] = max(s_count[1], cls); }
      }
      __syncthreads();
      const int cn = s_count[0];
      if (warp == 0) {
        // ------------------------------------------------------------- TMA producer
        if (elect_one()) {
          if (k0 == 0) { tma_prefetch_desc(&map_blocks); tma_prefetch_desc(&map_boxes); tma_prefetch_desc(&map_nodes); }
          for (int i = 0; i < cn && ok; ++i) {
            const int4 m = s_meta[i];
            const int nb = vtile_boxes(m.z), end = min(m.y, panel0 + RANGE);
            for (int j = panel0; j < end; j += 2) {
              if (!(ok = mbar_wait_thin(empty + 8 * st, st_ph ^ 1u, abort_flag))) break;
              // (a lone panel is followed by zeros from behind the last block: the accumulator's other half has to hold something)
              mbar_expect_tx(full + 8 * st, (uint32_t)(2 * nb * JOINT_ROWS * PANEL * 2));
              for (int p = 0; p < 2; ++p) {
                const uint32_t dst = sRing + st * TV_STAGE + p * TV_PANEL;
                const bool there = j + p < end, nodes = there && m.w < 0;
                const int y = nodes ? (req * v.NC + j + p) * TREE_PANEL_ROWS : there ? (m.w + j + p) * TILE : v.n_blocks * TILE;
                if (nb == TILE / JOINT_ROWS) {
                  tma_load_2d(dst, &map_blocks, full + 8 * st, 0, y);
                } else {
                  for (int b = 0; b < nb; ++b)
                    tma_load_2d(dst + b * (JOINT_ROWS * PANEL * 2), nodes ? &map_nodes : &map_boxes, full + 8 * st, 0, y + (there ? b * JOINT_ROWS : 0));
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
          for (int i = 0; i < cn && ok; ++i, ++k) {
            const int4 m = s_meta[i];
            const int nb = vtile_boxes(m.z), end = min(m.y, panel0 + RANGE);
            if (!(ok = mbar_wait_thin(p_full, k & 1u, abort_flag))) break;
            fence_after_sync();
            if (since >= a.drain) { touched = 0; since = 0; }      // the weight warps have emptied the accumulators
            since += nb;
            for (int j = panel0; j < end; j += 2) {
              if (!(ok = mbar_wait_thin(full + 8 * st, st_ph, abort_flag))) break;
              fence_after_sync();
              const uint32_t acc = (uint32_t)(j - panel0) >> 1, d = tmem_base + acc * 128, w = tmem_base + COL_P;
              constexpr uint32_t idesc = idesc_f16(BF16 ? 1 : 0, 128, 128) | (1u << 16);            // B MN-major
              const uint32_t b_lo = (((sRing + st * TV_STAGE) >> 4) & 0x3fffu) | ((TV_PANEL >> 4) << 16);
              uint32_t more = (touched >> acc) & 1u;
              auto step = [&](int p, int ks) {                  // one part of the weights of 16 tokens
                mma_f16_ts(d, w + 64 * p + 8 * ks, ((uint64_t)KMAJOR_SW128_DESC_HI << 32) | (b_lo + ks * 128u), idesc, more);
                more = 1u;
              };
              // the small parts of all tokens first: the sum is cut after every instruction
              if (nb == TILE / JOINT_ROWS) {                      // (a loop of its own: the checks would cost this thread its pace)
#pragma unroll
                for (int p = PARTS - 1; p >= 0; --p)
#pragma unroll
                  for (int ks = 0; ks < 8; ++ks) step(p, ks);
              } else {
#pragma unroll 1
                for (int p = PARTS - 1; p >= 0; --p)
#pragma unroll 1
                  for (int ks = 0; ks < nb; ++ks) step(p, ks);
              }
              touched |= 1u << acc;
              mma_commit(empty + 8 * st);
              if (++st == TV_STAGES) { st = 0; st_ph ^= 1u; }
            }
            if (!ok) break;
            mma_commit(p_done);
          }
        }
        __syncwarp();
      } else if (warp == 2) {
        // ------------------------------------------------------------- TMA producer of the scores, a tile ahead of the weights
        if (elect_one()) {
          if (k0 == 0) { tma_prefetch_desc(&map_scores); tma_prefetch_desc(&map_score_boxes); }
          for (int i = 0; i < cn && ok; ++i, ++k) {
            const int4 m = s_meta[i];
            const int nb = vtile_boxes(m.z);
            if (!(ok = mbar_wait_thin(sc_empty, (k & 1u) ^ 1u, abort_flag))) break;
            mbar_expect_tx(sc_full, (uint32_t)(nb * JOINT_ROWS * a.v_box * 4));
            if (nb == TILE / JOINT_ROWS) tma_load_2d(sScores, &map_scores, sc_full, c0, m.x * TILE);
            else
              for (int b = 0; b < nb; ++b) tma_load_2d(sScores + b * (uint32_t)(JOINT_ROWS * a.v_box * 4), &map_score_boxes, sc_full, c0, m.x * TILE + b * JOINT_ROWS);
          }
          if (!ok && k > 0) mbar_wait_drain(sc_full, (k - 1) & 1u);
        }
        __syncwarp();
      }
      __syncthreads();                                          // the descriptors may be replaced
      ok = ok && !*abort_flag;
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(TV_REGS_WEIGHTS));
    const int quarter = warp & 3, part = (warp - 4) >> 2, row = quarter * 32 + lane;      // query row, tokens 32 part .. + 31
    const bool in = c0 + row < a.C;
    const float scale = (v.sm_scale == 0.f ? 1.f : fabsf(v.sm_scale)) * TV_LOG2E;      // scores come without their scale; weights are powers of two
    const uint64_t scale2 = tv_pack(scale, scale);
    const uint32_t lanes = tmem_base + ((uint32_t)(quarter * 32) << 16);
    // Row of the partial results that this thread's column of the request stands for; -1: no node's.
    const int c = c0 + row, g = c / a.Rs, n = c - g * a.Rs, t = n / v.rep;
    const long long r = c < a.C && n < a.R && t < info.y ? ((long long)(req * a.T + t) * a.n_splits + split) * v.Hq + g * v.rep + n % v.rep : -1;
    // The tensor core cuts its fp32 sums after every instruction, so an accumulator's error grows with the tiles in it.  After `drain` boxes of sixteen tokens it is emptied,
    // its expected loss given back, onto the partial result in memory: `stored`, accumulators that have been; worth `kept` of what it was then.
    float* const out = a.part_acc + (size_t)(r < 0 ? 0 : r) * v.d_kv + panel0 * PANEL;
    const int col0 = part * (COLS / 4);
    uint32_t stored = 0;
    int since = 0;                                                // boxes of sixteen tokens in the accumulators
    // Instructions of this thread's tokens that cost the row's sums bits, sixteen bits per accumulator.  One costs nothing where the row's weights of its sixteen
    // tokens fit one part (all of a size, or zeros: the products are short and their sums exact) or lie 2^TV_SMALL below the largest (shifted out of
    // the sum instead of cutting it): a softmax that few tokens decide is summed without loss, and gets nothing back.
    constexpr int LOSSY = (RANGE / 2 + 1) / 2;
    uint32_t lossy[LOSSY] = {};
    float give[RANGE / 2];                                        // what the accumulators get back
    auto lost = [&]() {                                           // of all four parts, which have stored theirs
      uint32_t n[LOSSY];
#pragma unroll
      for (int i = 0; i < LOSSY; ++i) {
        const uint32_t* const p = s_lossy + i * 4 * TILE + row;
        n[i] = p[0] + p[TILE] + p[2 * TILE] + p[3 * TILE];
      }
#pragma unroll
      for (int e = 0; e < RANGE / 2; ++e) give[e] = 1.f + TREE_CUT_VALUES * (float)(n[e >> 1] >> 16 * (e & 1) & 0xffffu);
    };
    auto tell = [&]() {
#pragma unroll
      for (int i = 0; i < LOSSY; ++i) s_lossy[(4 * i + part) * TILE + row] = lossy[i];
    };
    float kept = 1.f, largest = 0.f;                              // of the partial result, as it is stored
    auto read_out = [&](int c, float (&o)[32]) {                 // 32 of this thread's columns of the partial result
#pragma unroll
      for (int b = 0; b < 32; b += 8)
        if (r >= 0 && ((stored >> ((c + b) >> 7)) & 1u)) tv_ld8(out + c + b, o + b);
    };
    auto empty_onto = [&](int c, float (&o)[32], float f) {       // and the accumulators' columns, times f, onto them
#pragma unroll
      for (int b = 0; b < 32; b += 8) {
        const uint32_t acc = (uint32_t)(c + b) >> 7;
        const bool held = (stored >> acc) & 1u, fresh = (touched >> acc) & 1u;
        if (!held && !fresh) continue;
        float fc = f;
#pragma unroll
        for (int e = 0; e < RANGE / 2; ++e)
          if (acc == (uint32_t)e) fc = f * give[e];
        float d[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (fresh) {
          tmem_ld8(lanes + c + b, reinterpret_cast<uint32_t*>(d));
          tmem_ld_wait();
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) d[e] = held ? o[b + e] * kept + d[e] * fc : d[e] * fc;
        if constexpr (!BF16) {
#pragma unroll
          for (int e = 0; e < 8; ++e) largest = fmaxf(largest, fabsf(d[e]));
        }
        if (r >= 0) tv_st8(out + c + b, d);
      }
    };
    float top = -INFINITY;
    uint64_t l_sum2 = 0;                                        // two sums of this thread's weights
    for (int k0 = 0; k0 < n_mine; k0 += TV_META) {
      __syncthreads();
      const int cn = s_count[0];
      for (int i = 0; i < cn; ++i, ++k) {
        const int4 m = s_meta[i];
        // rows of the tile that hold no token, and columns past the last, count as -inf
        float x[32];
        bool got = __all_sync(0xffffffffu, mbar_wait(sc_full, k & 1u, abort_flag));
        {
          const float* p = s_scores + part * 32 * a.v_box + row;
          const int left = in ? m.z - part * 32 : 0;
          if (left >= 32) {
#pragma unroll
            for (int u = 0; u < 32; ++u) x[u] = p[u * a.v_box];
          } else {
#pragma unroll
            for (int u = 0; u < 32; ++u) x[u] = u < left ? p[u * a.v_box] : -INFINITY;
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(sc_empty);                     // the next tile's may come
        // the tile's maximum of the row, from the four threads that share it
        float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};      // two of each sixteen tokens
#pragma unroll
        for (int u = 0; u < 16; u += 2)
#pragma unroll
          for (int e = 0; e < 4; ++e) mx[e] = fmaxf(mx[e], x[(e >> 1) * 16 + u + (e & 1)]);
        const float mx0 = fmaxf(mx[0], mx[1]), mx1 = fmaxf(mx[2], mx[3]);
        float* const sm = s_max + (k & 1u) * 4 * TILE + row;
        sm[part * TILE] = fmaxf(mx0, mx1);
        if (since >= a.drain) tell();
        // a wait that ran out in one warp ends the loop in the four of its quarter, here: none is left at a barrier
        if (!(ok = named_bar_and(1 + quarter, 128, ok && got))) break;
        const float most = fmaxf(fmaxf(sm[0], sm[TILE]), fmaxf(sm[2 * TILE], sm[3 * TILE])) * scale;
        const bool grow = most > top + (HEAD + 8.f);              // also the first finite maximum
        const float next = grow ? most - HEAD : top, f = next == top ? 1.f : tv_ex2(top - next);      // 0 where there was none yet
        top = next;
        const float ref = top == -INFINITY ? 0.f : top;           // (a node that sees nothing so far has no maximum: weights stay 0)
        const uint64_t nm2 = tv_pack(-ref, -ref);
        float la, lb;
        tv_unpack(l_sum2, la, lb);
        l_sum2 = tv_pack(la * f, lb * f);
        kept *= f;
        const bool any = part * 32 < vtile_boxes(m.z) * JOINT_ROWS;      // (the products leave the other tokens out)
        uint32_t w[PARTS][16];                                    // the largest part first
#pragma unroll
        for (int u = 0; u < 32; u += 2) {
          float x0, x1;
          tv_unpack(tv_fma2(tv_pack(x[u], x[u + 1]), scale2, nm2), x0, x1);
          const uint64_t p = tv_pack(tv_ex2(x0), tv_ex2(x1));
          l_sum2 = tv_add2(l_sum2, p);
          if constexpr (PARTS == 3) tree_split3(p, w[0][u >> 1], w[1][u >> 1], w[2][u >> 1]);
          else split_pair_16<BF16>(p, w[0][u >> 1], w[1][u >> 1]);
        }
        uint32_t low[2] = {0u, 0u};                               // second parts of each sixteen weights: zero, or not
#pragma unroll
        for (int u = 0; u < 16; ++u) low[u >> 3] |= w[1][u];
        const float small = top + (HEAD - TV_SMALL);
        const uint32_t cuts = (low[0] != 0u && mx0 * scale > small ? 1u : 0u) + (low[1] != 0u && mx1 * scale > small ? 1u : 0u);
        if (k > 0) {
          const bool full_up = since >= a.drain;
          float o[32];
          if (full_up) read_out(col0, o);
          ok = __all_sync(0xffffffffu, mbar_wait(p_done, (k - 1) & 1u, abort_flag));
          fence_after_sync();
          if (full_up && ok) {
            lost();
            empty_onto(col0, o, f);
#pragma unroll 1
            for (int c = col0 + 32; c < col0 + COLS / 4; c += 32) {
              read_out(c, o);
              empty_onto(c, o, f);
            }
            stored |= touched;
            touched = 0;
            since = 0;
            kept = 1.f;
#pragma unroll
            for (int i = 0; i < LOSSY; ++i) lossy[i] = 0u;
          } else if (__any_sync(0xffffffffu, grow) && ok) {
            // seldom: this part's columns of the accumulators take the rows' factors
#pragma unroll 1
            for (int c = col0; c < col0 + COLS / 4; c += 8) {
              if (!((touched >> (c >> 7)) & 1u)) continue;
              uint32_t o[8];
              tmem_ld8(lanes + c, o);
              tmem_ld_wait();
#pragma unroll
              for (int e = 0; e < 8; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
              tmem_st8(lanes + c, o);
            }
          }
        }
        since += vtile_boxes(m.z);
        if (!ok) continue;
        const int reach = (min(m.y, panel0 + RANGE) - panel0 + 1) >> 1;
        // two parts of sixteen tokens are two instructions (those of three bf16 parts: see TREE_CUT_VALUES); the small parts of an accumulator's first tile
        // come before its sum has its size
#pragma unroll
        for (int e = 0; e < RANGE / 2; ++e)
          if (e < reach) lossy[e >> 1] += cuts << (16 * (e & 1) + (int)((touched >> e) & 1u));
        touched |= (1u << reach) - 1u;
        if (any) {
#pragma unroll
          for (int p = 0; p < PARTS; ++p) tmem_st16(lanes + COL_P + 64 * p + 16 * part, w[p]);
        }
        tmem_st_wait();
        fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_full);
      }
      __syncthreads();                                          // the descriptors may be replaced
      ok = ok && !*abort_flag;
    }
    // ----------------------------------------------------------- partial results of this split
    float la, lb;
    tv_unpack(l_sum2, la, lb);
    s_max[part * TILE + row] = la + lb;                         // (behind the loop's last __syncthreads: nobody reads maxima any more)
    tell();
    if (ok && k > 0) ok = __all_sync(0xffffffffu, mbar_wait(p_done, (k - 1) & 1u, abort_flag));
    fence_after_sync();
    named_bar_sync(1 + quarter, 128);
    // This part's columns, a row per thread; columns that no tile reached are left alone, as is everything where no tile reached the range: the
    // merge knows it from the split's widest class.
    largest = 0.f;
    if (ok && k > 0) {
      lost();
#pragma unroll 1
      for (int c = col0; c < col0 + COLS / 4; c += 32) {
        float o[32];
        read_out(c, o);
        empty_onto(c, o, 1.f);
      }
    }
    if constexpr (!BF16) {
      s_max[(4 + part) * TILE + row] = largest;
      named_bar_sync(1 + quarter, 128);
    }
    if (part == 0 && r >= 0) {
      if constexpr (!BF16) {
        const float* const b = s_max + 4 * TILE + row;
        reinterpret_cast<float*>(a.part_x + r)[range] = fmaxf(fmaxf(b[0], b[TILE]), fmaxf(b[2 * TILE], b[3 * TILE]));
      }
      reinterpret_cast<float*>(a.part_m + r)[range] = top;
      if (range == 0) a.part_l[r] = (s_max[row] + s_max[TILE + row]) + (s_max[2 * TILE + row] + s_max[3 * TILE + row]);
    }
    tmem_ld_wait();
  }
  if (tid == 0 && range == 0 && blockIdx.y == 0) a.part_cls[req * a.n_splits + split] = s_count[1];
  fence_before_sync();
  __syncthreads();
  fence_after_sync();
  if (warp == 1) tmem_dealloc(tmem_base, 512);
  if (tid == 0 && *abort_flag) set_status(v, misaligned ? TWKV_ERR_DEVICE_CHECK : TWKV_ERR_TIMEOUT);
}

cudaError_t launch_tree_value(const DevView& v, const TreeCall& a, const TreeMaps& maps, cudaStream_t st) {
  ProfScope ps(TWKV_K_VACC, st);
  auto kernel = v.dtype != TWKV_BF16 ? tree_value_kernel<false, 2> : a.n_parts == 3 ? tree_value_kernel<true, 3> : tree_value_kernel<true, 2>;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)TV_SMEM);
  if (e != cudaSuccess) return e;
  e = launch_chained(kernel, dim3(a.n_req * a.n_splits, (a.C + TILE - 1) / TILE, (v.NC + a.range - 1) / a.range), dim3(TV_THREADS), dim3(1), TV_SMEM, st,
                     maps.blocks, maps.boxes, maps.node_boxes, maps.scores, maps.score_boxes, v, a);
  if (e != cudaSuccess) return e;
  count_launch();
  return cudaGetLastError();
}

}  // namespace twkv
