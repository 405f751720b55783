// One launch prepares a pass of tree attention; its CTAs are, in this order:
//   NC       one per rank class: the class's entries of the K list
//   n_req    the splits of a request's V tiles
//   n_req vj K slot -> score row of its cached tokens; the first also the tables of its joint tiles
//   n_req 2  the nodes' states cut to their ranks, as a tile of keys and a tile of values
//   n_req qc its queries as the operand of the score products
// The K list holds a request's tiles together, from the widest class to the narrowest, in items of two: a pair of CTAs rebuilds two
// tiles at once and multiplies them with the same queries, so both belong to one request; the narrower one's missing panels are zeros.
// A request with an odd number of tiles ends with a filler.  Where a class's entries of a request start follows from the keys' token
// counts, as in a decode pass; the order of tiles of one class inside a request depends on timing, and no result does.
// What bounds it is the depth of its dependent reads and scans: 8 us and the launch for one request, 29 for 64 (one CTA of 1024 threads per SM, 500 CTAs).
#include <algorithm>
#include <climits>

#include "twkv_dev.h"
#include "mma_util.cuh"
#include "scan_util.cuh"
#include "joint_tiles.cuh"
#include "tree.h"

namespace twkv {

// Estimated cycles of an item of the score kernel: per KV head and pass a part for rotation and score products, which grow with the query rows, beyond
// 64 with the stores of the scores; and a part per panel, more of it where the panels are brought once per KV head.  Fitted to lists of one class
// (16 to 512 query rows, 1 to 16 panels).  Only the ratios matter.
__device__ __forceinline__ unsigned tree_cost(const DevView& v, const TreeCall& a, int cls) {
  const unsigned rows = 14u * (unsigned)min(a.R, 64) + 28u * (unsigned)max(a.R - 64, 0);
  if (cls <= 8) return (unsigned)v.Hkv * (1500u + rows + 300u * (unsigned)cls);
  if (a.R > 64) return (unsigned)v.Hkv * (1500u + rows + 500u * (unsigned)cls);
  return (unsigned)v.Hkv * (3000u + 3u * rows + 300u * (unsigned)cls);
}

// Refuses a request whose sequence an earlier one names, or into whose rows an earlier one reaches: those are not its to write (the
// whole CTA asks; the result is valid for all threads).
__device__ __forceinline__ int4 tree_distinct(const TreeCall& a, int i, int4 r) {
  int seq = 0, row = 0;
  for (int j = threadIdx.x; j < a.r0 + i; j += blockDim.x) {
    seq |= a.req_seqs[j] == r.z;
    row |= a.offsets[j] > r.x;
  }
  if (__syncthreads_or(seq)) r.z = -1;
  if (__syncthreads_or(row)) { r.z = -1; r.y = 0; }
  return r;
}

// Largest value of the threads before this one (INT_MIN: none) over a CTA of 1024 threads; *total = the largest of all.
__device__ __forceinline__ int block_max_excl(int x, int* s_warp, int* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int incl = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int u = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl = max(incl, u);
  }
  __syncthreads();
  if (lane == 31) s_warp[warp] = incl;
  __syncthreads();
  int before = INT_MIN, all = INT_MIN;
  for (int w = 0; w < 32; ++w) {
    const int m = s_warp[w];
    if (w < warp) before = max(before, m);
    all = max(all, m);
  }
  const int prev = __shfl_up_sync(0xffffffffu, incl, 1);
  *total = all;
  return lane ? max(before, prev) : before;
}

// What a warp finds about request i, apart from repeated sequences: first row, nodes, sequence (-1: refused), classes of the nodes'
// tiles (K | V << 8).
__device__ __forceinline__ int4 tree_request(const DevView& v, const TreeCall& a, int i) {
  const int lane = threadIdx.x & 31;
  int first, n;
  bool ok = tree_rows(a.offsets, a.r0 + i, a.n_rows, a.T, &first, &n);
  const int seq = a.req_seqs[a.r0 + i];
  ok = ok && seq >= 0 && seq < v.S;
  unsigned rk = 0u, rv = 0u;
  for (int j = lane; j < n; j += 32) {
    const unsigned w = reinterpret_cast<const unsigned*>(a.levels)[first + j];
    const int pos = a.positions[first + j];
    const unsigned k = w & 0xffffu, x = w >> 16;
    ok = ok && k >= 1u && k <= (unsigned)v.d_kv && x >= 1u && x <= (unsigned)v.d_kv && pos >= 0 && pos < ROPE_LO * ROPE_HI;
    rk = max(rk, k); rv = max(rv, x);
  }
  ok = __all_sync(0xffffffffu, ok);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) { rk = max(rk, __shfl_xor_sync(0xffffffffu, rk, o)); rv = max(rv, __shfl_xor_sync(0xffffffffu, rv, o)); }
  return make_int4(first, n, ok ? seq : -1, (int)((rk + PANEL - 1) / PANEL | (rv + PANEL - 1) / PANEL << 8));
}

// K tiles of a request in class k + 1: its own, less those that lie in joint tiles, the joint tiles that start there, and the nodes'.
__device__ __forceinline__ int tree_tiles(int fill, unsigned joint, int k, int node_cls) {
  return fill / TILE + (fill % TILE != 0 && !((joint >> (16 + k)) & 1u) ? 1 : 0) + (int)((joint >> k) & 1u) + (node_cls == k + 1 ? 1 : 0);
}

struct TreeSmem {          // of the class CTAs, behind one another in dynamic shared memory
  int *first;              // [S] first request of the call that names the sequence
  int *base, *cur;         // [n_req] first entry of the request (tiles of the request until it is known), next entry of this class
  int* mine;               // [n_req] tiles in this class
  int *node;               // [n_req] class of the nodes' keys, 0: the request has no entries
  unsigned* joint;         // [n_req]
  unsigned long long* cost;    // [n_req + 1] (first class CTA) estimated cost of the requests before
};
static size_t tree_plan_smem(int S, int n_req) { return (size_t)S * 4 + (size_t)n_req * 20 + (size_t)(n_req + 2) * 8 + 16; }

__device__ void tree_klist(const DevView& v, const TreeCall& a, int layer, int n_pieces) {
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ int s_warp[32];
  __shared__ unsigned s_wide;
  __shared__ int s_hg;
  TreeSmem s;
  s.cost = reinterpret_cast<unsigned long long*>(smem);
  s.first = reinterpret_cast<int*>(s.cost + a.n_req + 2);
  s.base = s.first + v.S; s.cur = s.base + a.n_req; s.mine = s.cur + a.n_req; s.node = s.mine + a.n_req; s.joint = reinterpret_cast<unsigned*>(s.node + a.n_req);
  const int NC = v.NC, run = blockIdx.x, cls = NC - run, tid = threadIdx.x, warp = tid >> 5;
  const int* fill = v.fill_l(layer);
  // the first of this class's tiles, used at the end
  const int n_list = v.kcc(layer)[cls - 1];
  const int4* desc = v.desc(layer, 0);
  const int* list = v.kct(layer) + (size_t)(cls - 1) * v.NT;
  int tile = 0;
  int4 d = make_int4(0, 0, 0, 0);
  if (tid < n_list) {
    tile = list[tid];
    d = desc[tile];
  }
  for (int i = tid; i < v.S; i += 1024) s.first[i] = 0x7fffffff;
  if (tid == 0) s_wide = 0u;
  __syncthreads();
  for (int i0 = 0, most = INT_MIN; i0 < a.r0 + a.n_req; i0 += 1024) {
    const int i = i0 + tid;
    const bool in = i < a.r0 + a.n_req;
    const int seq = in ? a.req_seqs[i] : -1, off = in ? a.offsets[i] : INT_MIN;
    if (seq >= 0 && seq < v.S) atomicMin(&s.first[seq], i);
    int all = INT_MIN, before = INT_MIN;
    if (a.r0 + a.n_req > 1) before = max(most, block_max_excl(off, s_warp, &all));
    most = max(most, all);
    if (in && i >= a.r0) s.cur[i - a.r0] = before > off;            // an earlier request reaches into this one's rows
  }
  __syncthreads();
  // a warp per request, a lane per class
  for (int i = warp; i < a.n_req; i += 32) {
    const int4 r = tree_request(v, a, i);
    const int lane = tid & 31, k = lane;
    const int node = r.z >= 0 && r.y > 0 && s.first[r.z] == a.r0 + i && !s.cur[i] ? r.w & 0xff : 0;
    unsigned joint = 0u, cost = 0u;
    int c = 0, before = 0;
    if (node) {
      joint = joint_masks(v, layer, r.z);
      c = k < NC ? tree_tiles(fill[(size_t)r.z * NC + k], joint, k, node) : 0;
      before = c;                                                  // tiles in this class and wider ones
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int u = __shfl_down_sync(0xffffffffu, before, o);
        if (lane + o < 32) before += u;
      }
      if (run == 0) {
        const int items = (before + 1) / 2 - (before - c + 1) / 2;  // whose wider tile has this class
        cost = items ? tree_cost(v, a, k + 1) : 0u;
        const unsigned wide = __reduce_max_sync(0xffffffffu, cost);
        if (lane == 0) atomicMax(&s_wide, wide);
        cost = __reduce_add_sync(0xffffffffu, cost * (unsigned)items);     // (2^20 tokens of eight heads are below 2^31)
      }
    }
    __syncwarp();
    if (lane == 0) {
      s.node[i] = node;
      s.joint[i] = joint;
      s.base[i] = before;                                          // all of them
      if (run == 0) s.cost[i] = cost;
    }
    if (lane == cls - 1) { s.cur[i] = before - c; s.mine[i] = c; }
  }
  __syncthreads();
  int base = 0;
  for (int i0 = 0; i0 < a.n_req; i0 += 1024) {
    const int i = i0 + tid;
    const int all = i < a.n_req ? s.base[i] : 0;
    int total;
    const int at = base + block_scan_excl((all + 1) & ~1, s_warp, &total);
    base += total;
    if (i < a.n_req) {
      const int wide = s.cur[i];
      s.base[i] = at;
      s.cur[i] = at + wide;
      if (s.node[i] == cls) {                                      // the nodes' tile, last of its class, and the filler
        const int seq = a.req_seqs[a.r0 + i], n = a.offsets[a.r0 + i + 1] - a.offsets[a.r0 + i];
        a.klist[at + wide + s.mine[i] - 1] = make_int4(i * (v.TPS + 1) + v.svc(layer)[seq], cls | TREE_NODES | n << 16, i * NC * TREE_PANEL_ROWS, i);
        if (all & 1) a.klist[at + all] = make_int4(0, TREE_FILLER, 0, i);
      }
    }
  }
  __syncthreads();
  // this class's tiles
  for (int i = tid; i < n_list; i += 1024) {
    if (i != tid) {
      tile = list[i];
      d = desc[tile];
    }
    const int slot = s.first[d.x] - a.r0;
    if (slot < 0 || slot >= a.n_req || s.node[slot] == 0) continue;
    if (d.z < TILE && ((s.joint[slot] >> (15 + cls)) & 1u)) continue;                    // lies in a joint tile
    a.klist[atomicAdd(&s.cur[slot], 1)] = make_int4(tile, d.y | d.z << 16, d.w, slot);
  }
  for (int i = tid; i < a.n_req; i += 1024) {
    const unsigned j = s.joint[i];
    if (s.node[i] && ((j >> (cls - 1)) & 1u))
      a.klist[atomicAdd(&s.cur[i], 1)] = make_int4(~(i * (NC / 2) + __popc((j & 0xffffu) >> cls)), cls | TILE << 16, 0, i);
  }
  if (run > 0) return;
  // costs of the requests before, and the parts an item's KV heads are dealt out in (the estimate of a decode pass)
  if (warp == 0) {
    unsigned long long sum = 0ull;
    for (int i0 = 0; i0 < a.n_req; i0 += 32) {
      const int i = i0 + tid;
      const unsigned long long mine = i < a.n_req ? s.cost[i] : 0ull;
      unsigned long long incl = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const unsigned long long u = __shfl_up_sync(0xffffffffu, incl, o);
        if (tid >= o) incl += u;
      }
      if (i < a.n_req) s.cost[i] = sum + incl - mine;
      sum += __shfl_sync(0xffffffffu, incl, 31);
    }
    if (tid == 0) {
      s.cost[a.n_req] = sum;
      const int items = base / 2;
      const float part_cost = 2600.f, per = 1.f / (float)n_pieces, wide = (float)s_wide;
      float best = 3.4e38f, part = 1.f;
      int hg = 1;
      for (int h = 1; v.Hkv % h == 0; h *= 2, part *= 0.5f) {
        const float est = items * h <= n_pieces ? wide * part : ((float)sum + (float)items * (float)(h - 1) * part_cost) * per + 0.7f * wide * part;
        if (est < best) { best = est; hg = h; }
      }
      s_hg = hg;
      *a.parts = hg;
      a.cta_start[n_pieces] = items * hg;
    }
  }
  __syncthreads();
  const int hg = s_hg;
  const unsigned long long total = s.cost[a.n_req], per_piece = total / (unsigned)n_pieces;
  const unsigned over = (unsigned)(total - per_piece * (unsigned)n_pieces);
  for (int b = tid; b < n_pieces; b += 1024) {
    int start = 0;
    if (total > 0ull) {
      const unsigned long long key = (unsigned long long)b * per_piece + (unsigned)b * over / (unsigned)n_pieces;      // total b / n_pieces
      int lo = 0, hi = a.n_req - 1;                                // the last request whose cost starts at or before the key
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (s.cost[mid] <= key) lo = mid; else hi = mid - 1;
      }
      const int node = s.node[lo], seq = node ? a.req_seqs[a.r0 + lo] : 0;
      const unsigned joint = s.joint[lo];
      int tokens[TWKV_MAX_CLASSES];                                // (read at once)
#pragma unroll
      for (int k = 0; k < TWKV_MAX_CLASSES; ++k) tokens[k] = k < NC && node ? fill[(size_t)seq * NC + k] : 0;
      unsigned rest = (unsigned)(key - s.cost[lo]), within = 0u;
      int all = 0, item = 0;
#pragma unroll
      for (int k = TWKV_MAX_CLASSES - 1; k >= 0; --k) {
        if (k >= NC || !node) continue;
        const int c = tree_tiles(tokens[k], joint, k, node);
        const int items = (all + c + 1) / 2 - (all + 1) / 2;
        const unsigned one = tree_cost(v, a, k + 1);
        if (rest < (unsigned)items * one) {
          within = rest / (one / (unsigned)hg);                    // (hg parts the KV heads, so it divides an item's cost)
          break;
        }
        rest -= (unsigned)items * one;
        item += items;
        all += c;
      }
      start = (s.base[lo] / 2 + item) * hg + (int)within;
    }
    a.cta_start[b] = start;
  }
}

constexpr float TREE_CTA_COST = 200.f;
// Estimated time of the value kernel and the merge with s splits, all requests taken to be like this one; in the time of a panel's product with a
// sixteen-token box (44 ns).  work: of a request's tiles, per range of panels.  A CTA costs as much as four tiles before and behind them, CTAs come to the SMs
// as these get free, and the merge reads every split's sums at 3 TB/s.  Value kernel and merge in us by splits, the choice last: 16 sequences of 2048
// tokens, 8 nodes: 1: 79, 2: 64, 4: 76, 2; 20 of 3000, 4 nodes: 1: 114, 3: 80, 7: 107, 2 or 3; one of 16384, 16 nodes: 8: 70, 16: 61, 32: 81, 16; 8 of 4096: 2: 74,
// 4: 61, 9: 79, 3; one of 65536, 4 nodes: 16: 94, 64: 71, 32 to 64.
__device__ __forceinline__ float tree_splits_cost(const DevView& v, const TreeCall& a, const int* work, int sms, int s) {
  const float groups = (float)(a.n_req * ((a.C + TILE - 1) / TILE)), inv = 1.f / (float)s;
  float all = 0.f, longest = 0.f;
  int panels = 0;
  for (int z = 0; z < TREE_MAX_RANGES; ++z) {
    if (work[z] == 0) continue;
    all += (float)work[z] + TREE_CTA_COST * (float)s;
    longest = fmaxf(longest, (float)work[z] * inv + TREE_CTA_COST);
    panels += a.range;
  }
  const float bytes = (float)(a.n_req * a.T * v.Hq) * (float)(min(panels, v.NC) * PANEL * 4);
  return fmaxf(longest, groups * all / (float)sms + 0.3f * longest) + (float)s * (8.f + bytes * 7.5e-6f);
}

// vtile_stride() by a warp, a candidate per lane: of 32 numbers behind one another one is always coprime to n (there are at most 25 between two such,
// up to 510510).  The search one after the other took 2000 to 5000 cycles.
__device__ __forceinline__ int tree_stride(int n) {
  if (n < 3) return 1;
  const int first = max((int)(((long long)n * 618034ll) / 1000000ll), 1);
  int x = first + (int)(threadIdx.x & 31), y = n;
  while (y) { const int t = x % y; x = y; y = t; }
  return first + __ffs(__ballot_sync(0xffffffffu, x == 1)) - 1;
}

static_assert(TREE_MAX_SPLITS == 64, "two warps");
// Cut points of a request's V tiles, the nodes' last, into splits of about equal cost, as for a decode pass.
__device__ void tree_vsplit(const DevView& v, const TreeCall& a, int layer, int i, const int4& r, int sms) {
  __shared__ int s_warp[32], s_work[TREE_MAX_RANGES];
  __shared__ uint2 s_best[TREE_MAX_SPLITS / 32];
  const int tid = threadIdx.x, n_splits = a.n_splits;
  int* cut = a.vcut + (size_t)i * (n_splits + 1);
  const int nv = r.z >= 0 && r.y > 0 ? v.svc(layer)[r.z] : 0, n = r.z >= 0 && r.y > 0 ? nv + 1 : 0;
  if (n == 0) {
    if (tid == 0) a.info[i] = make_int4(r.x, r.y, r.z, 0);
    for (int s = tid; s <= n_splits; s += 1024) cut[s] = 0;
    return;
  }
  if (tid < TREE_MAX_RANGES) s_work[tid] = 0;
  __syncthreads();                                                 // before any warp adds to it
  const int* list = v.svt(layer) + (size_t)r.z * v.TPS;
  const int4* desc = v.desc(layer, 1);
  const int stride = tree_stride(nv);
  int4* meta = a.vmeta + (size_t)i * (v.TPS + 1);
  auto cost = [&](int k, bool count) -> int {
    if (k >= n) return 0;
    int4 m;
    if (k < nv) {
      const int at = vtile_at(k, stride, nv);
      const int4 d = desc[list[at]];
      m = make_int4(i * (v.TPS + 1) + at, d.y, d.z, d.w);
    } else {
      m = make_int4(i * (v.TPS + 1) + nv, r.w >> 8, r.y, -1);
    }
    meta[k] = m;
    // in panels' products: a tile's weights take as long as those of four panels; wide tiles are taken in ranges, by CTAs of their own
    auto of_range = [&](int z) { return m.y > z * a.range ? vtile_boxes(m.z) * max(min(m.y - z * a.range, a.range), 4) + 4 : 0; };
    if (count)
      for (int z = 1; z < TREE_MAX_RANGES && m.y > z * a.range; ++z) atomicAdd(&s_work[z], of_range(z));
    return of_range(0);
  };
  int total = 0, w = 0, off = 0;                                   // this thread's last tile: cost, cost of those before
  for (int k0 = 0; k0 < n; k0 += 1024) {
    int part;
    w = cost(k0 + tid, true);
    off = total + block_scan_excl(w, s_warp, &part);
    total += part;
  }
  if (tid == 0) s_work[0] = total;
  __syncthreads();
  if (tid < TREE_MAX_SPLITS) {                                      // two warps, a number of splits per thread; of equal ones the smaller
    const unsigned est = tid < min(n_splits, n) ? __float_as_uint(tree_splits_cost(v, a, s_work, sms, tid + 1)) : 0xffffffffu;      // (positive)
    const unsigned least = __reduce_min_sync(0xffffffffu, est), who = __ballot_sync(0xffffffffu, est == least);
    if ((tid & 31) == 0) s_best[tid >> 5] = make_uint2(least, tid + __ffs(who));
  }
  __syncthreads();
  const int used = (int)(s_best[1].x < s_best[0].x ? s_best[1].y : s_best[0].y);
  if (tid == 0) a.info[i] = make_int4(r.x, r.y, r.z, used);
  const unsigned W = (unsigned)total, ns = (unsigned)used;          // (4113 tiles of at most 52, 64 splits: far from 32 bits)
  int base = 0;
  for (int k0 = 0; k0 < n; k0 += 1024) {
    if (n > 1024) {
      int part;
      w = cost(k0 + tid, false);
      off = base + block_scan_excl(w, s_warp, &part);
      base += part;
    }
    if (k0 + tid < n) {
      const unsigned e = (unsigned)off, p = e + (unsigned)w;
      for (unsigned s = (e * ns + W - 1u) / W; s < ns && s * W / ns < p; ++s) cut[s] = k0 + tid;
    }
  }
  for (int s = used + tid; s <= n_splits; s += 1024) cut[s] = n;
}

// The nodes' states of one side, cut to their ranks, as panels [64 rows][64 components]; rows up to the next multiple of sixteen are
// zeros.  A value that is not finite would reach every query of the request through its weight 0: zeros stand for it, and the queries that
// see its node get what is not a number in the end.
template <bool BF16>
__device__ void tree_pack(const DevView& v, const TreeCall& a, int i, const int4& r, int side) {
  __shared__ unsigned long long s_bad;
  const int tid = threadIdx.x;
  if (tid == 0) s_bad = 0ull;
  __syncthreads();
  if (r.z >= 0) {
    const int cls = side ? r.w >> 8 : r.w & 0xff, rows = (r.y + 15) & ~15, pieces = cls * 8;
    const unsigned short* x = (side ? a.V : a.K) + (size_t)r.x * v.d_kv;
    unsigned char* out = (side ? a.nv : a.nk) + (size_t)i * v.NC * TREE_PANEL_ROWS * PANEL * 2;
    for (int k = tid; k < rows * pieces; k += 1024) {
      const int row = k / pieces, e = k - row * pieces;              // eight components from 8 e on
      uint4 w = make_uint4(0u, 0u, 0u, 0u);
      if (row < r.y) {
        const int keep = (int)a.levels[2 * (size_t)(r.x + row) + side] - 8 * e;
        if (keep > 0) w = *reinterpret_cast<const uint4*>(x + (size_t)row * v.d_kv + 8 * e);
        unsigned p[4] = {w.x, w.y, w.z, w.w};
        bool bad = false;
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          if (keep <= 2 * b) p[b] = 0u;
          else if (keep == 2 * b + 1) p[b] &= 0xffffu;
          constexpr unsigned inf = BF16 ? 0x7f80u : 0x7c00u;
          bad |= (p[b] & inf) == inf || ((p[b] >> 16) & inf) == inf;
        }
        if (side && bad) {
          atomicOr(&s_bad, 1ull << row);
          p[0] = p[1] = p[2] = p[3] = 0u;
        }
        w = make_uint4(p[0], p[1], p[2], p[3]);
      }
      reinterpret_cast<uint4*>(out + ((size_t)(e >> 3) * TREE_PANEL_ROWS + row) * (PANEL * 2))[e & 7] = w;
    }
  }
  __syncthreads();
  if (side && tid == 0) a.bad[i] = s_bad;
  if (!side && tid < 32) {                                           // the masks turned: a lane's two nodes' masks, one ballot per node seen
    const unsigned long long m0 = tid < r.y ? a.masks[r.x + tid] : 0ull, m1 = tid + 32 < r.y ? a.masks[r.x + tid + 32] : 0ull;
    for (int k = 0; k < TWKV_TREE_MAX_NODES; ++k) {
      const unsigned lo = __ballot_sync(0xffffffffu, (m0 >> k) & 1ull), hi = __ballot_sync(0xffffffffu, (m1 >> k) & 1ull);
      if (tid == 0) a.seers[(size_t)i * TWKV_TREE_MAX_NODES + k] = (unsigned long long)hi << 32 | lo;
    }
  }
}

// Queries of a request as f16 rows in the order in which the rotated keys are contracted: 16-byte piece 8 hf + 2 c holds dimensions
// 32 hf + 8 c .. + 7, piece 8 hf + 2 c + 1 the dimensions 64 above them.  Rows that no query has are zeros.
template <bool BF16>
__device__ void tree_queries(const DevView& v, const TreeCall& a, int i, const int4& r, int part, int parts) {
  const int tid = part * 1024 + threadIdx.x, step = parts * 1024;
  uint4* out = reinterpret_cast<uint4*>(a.qop + (size_t)i * v.Hkv * a.Rp * HEAD_DIM);
  // a negative scale goes into the queries, a zero one zeroes them (-inf masks need a positive factor)
  const unsigned flip = v.sm_scale < 0.f ? 0x80008000u : 0u, keep = v.sm_scale == 0.f ? 0u : 0xffffffffu;
  bool over = false;
  for (int k = tid; k < v.Hkv * a.Rp * 16; k += step) {
    const int kc = k & 15, row = k >> 4, g = row / a.Rp, n = row - g * a.Rp, t = n / v.rep;
    const int ch = (kc >> 3) * 4 + ((kc & 7) >> 1) + 8 * (kc & 1);
    uint4 w = make_uint4(0u, 0u, 0u, 0u);
    if (n < a.R && t < r.y) w = reinterpret_cast<const uint4*>(a.q + ((size_t)(r.x + t) * v.Hq + g * v.rep + n % v.rep) * HEAD_DIM)[ch];
    if constexpr (BF16) {
      const unsigned p[4] = {w.x, w.y, w.z, w.w};
      unsigned o[4];
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const float lo = __uint_as_float(p[b] << 16), hi = __uint_as_float(p[b] & 0xffff0000u);
        over |= !(fabsf(lo) <= 65504.f) || !(fabsf(hi) <= 65504.f);
        asm("cvt.rn.satfinite.f16x2.f32 %0, %1, %2;" : "=r"(o[b]) : "f"(hi), "f"(lo));
      }
      w = make_uint4(o[0], o[1], o[2], o[3]);
    }
    out[k] = make_uint4((w.x ^ flip) & keep, (w.y ^ flip) & keep, (w.z ^ flip) & keep, (w.w ^ flip) & keep);
  }
  if (over) set_status(v, TWKV_ERR_DEVICE_CHECK);                   // a bf16 query beyond the f16 range would be clamped
}

// K slot -> score row of a request's cached tokens: CTA j of vj takes eight of the sequence's V tiles at a time.
__device__ void tree_links(const DevView& v, const TreeCall& a, int layer, int i, const int4& r, int j, int vj) {
  const int n = v.svc(layer)[r.z];
  const int* list = v.svt(layer) + (size_t)r.z * v.TPS;
  const int4* desc = v.desc(layer, 1);
  const int* aux = v.aux(layer, 1);
  const int sub = threadIdx.x >> 7, slot = threadIdx.x & (TILE - 1);
  for (int t = j * 8 + sub; t < n; t += vj * 8) {
    const int vt = list[t];
    if (slot < desc[vt].z) v.kv_link[aux[(size_t)vt * TILE + slot]] = (i * (v.TPS + 1) + t) * TILE + slot;
  }
}

__global__ void __launch_bounds__(1024) tree_plan_kernel(DevView v, TreeCall a, int layer, int n_pieces, int vj, int qc, int sms) {
  __shared__ int4 s_r;
  chain_start();
  chain_wait();
  int b = blockIdx.x;
  if (b < v.NC) { tree_klist(v, a, layer, n_pieces); return; }
  b -= v.NC;
  // the request of a CTA: one job after the other, each for all requests
  const int n = a.n_req, per[4] = {1, vj, 2, qc};
  int job = 0;
  while (b >= n * per[job]) b -= n * per[job++];
  const int i = b / per[job], part = b % per[job];
  if (threadIdx.x < 32) {
    const int4 q = tree_request(v, a, i);
    if (threadIdx.x == 0) s_r = q;
  }
  __syncthreads();
  const int4 r = tree_distinct(a, i, s_r);
  if (job == 0) {
    if (r.z < 0 && threadIdx.x == 0) set_status(v, TWKV_ERR_INVALID_ARG);
    tree_vsplit(v, a, layer, i, r, sms);
  } else if (job == 1) {
    if (r.z < 0) return;
    tree_links(v, a, layer, i, r, part, vj);
    if (part > 0 || threadIdx.x >= TWKV_MAX_CLASSES / 2 * 32) return;
    const unsigned masks = joint_masks(v, layer, r.z);
    unsigned starts = masks & 0xffffu;
    for (int w = threadIdx.x >> 5; w > 0 && starts; --w) starts ^= 1u << (31 - __clz(starts));
    if (starts) joint_tile(v, layer, r.z, masks, 31 - __clz(starts), i * (v.NC / 2) + (threadIdx.x >> 5));
  } else if (job == 2) {
    if (v.dtype == TWKV_BF16) tree_pack<true>(v, a, i, r, part); else tree_pack<false>(v, a, i, r, part);
  } else {
    if (v.dtype == TWKV_BF16) tree_queries<true>(v, a, i, r, part, qc); else tree_queries<false>(v, a, i, r, part, qc);
  }
}

cudaError_t launch_tree_plan(const DevView& v, const TreeCall& a, int layer, int n_pieces, int sm_count, cudaStream_t st) {
  ProfScope ps(TWKV_K_PLAN, st);
  const int vj = a.n_req >= 128 ? 1 : std::min(std::min(64, (v.TPS + 7) / 8), (256 - a.n_req) / a.n_req);      // (a CTA takes eight tiles at a time)
  const int qc = std::max(1, std::min(8, v.Hkv * a.Rp * 16 / 4096));
  const size_t smem = tree_plan_smem(v.S, a.n_req);
  cudaError_t e = cudaFuncSetAttribute(tree_plan_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  e = launch_chained(tree_plan_kernel, dim3(v.NC + a.n_req * (3 + vj + qc)), dim3(1024), dim3(1), smem, st, v, a, layer, n_pieces, vj, qc, sm_count);
  if (e != cudaSuccess) return e;
  count_launch();
  return cudaGetLastError();
}

}  // namespace twkv
